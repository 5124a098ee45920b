// 8-bit floating-point codes with a scale for each block of 128: 1 x 128 values of a row (activations) or 128 x 128 of a matrix
// (weights).
//
//   m = max |x| over the block,   q = the E4M3 value nearest to 448 x / m (ties to the even code),   scale = m / 448
//
// The codes are rounded exactly.  With x = P 2^t, m = M 2^s and integers P, M < 256 the quotient is 7 P / M times a power of two,
// and what lies between two codes is B times one with an odd B <= 31.  Either the quotient is that border, or it is at least
// 1 / (31 * 255) = 1.26e-4 of it away (the difference of the integers 7 P 2^a and B M 2^b is one at least).  fp32's x * (448 / m)
// is off by 2^-23 of its value, and rounded to 13 fraction bits (6.1e-5) it falls on the border it belongs on and on no other.
//
// Bound by the bytes that cross HBM: three per value.
#include <cuda_fp8.h>

#include <algorithm>

#include "entry.cuh"
#include "spice_internal.cuh"

namespace spice {

namespace {

struct BlockArgs {
    const __nv_bfloat16 *w;   // [count, rows, cols]
    uint8_t *q;               // the same
    float *scale;             // [count, row blocks, column blocks]
    int64_t blocks;           // rows of blocks in all: count * rows, or count * ceil(rows / 128)
    int32_t rows, cols, kb;   // kb: blocks of a row
};

__device__ __forceinline__ uint4 load16(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// largest magnitude as bf16 bits: they compare like integers
__device__ __forceinline__ uint32_t largest(uint4 v) {
    const uint32_t a = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(a & 0xffffu, a >> 16);
}

// What turns the values of a block with largest magnitude m (bf16 bits) into codes
struct BlockScale {
    float pre, r;   // x * pre * r; pre lifts blocks whose 448 / m is beyond fp32
    bool finite;
    __device__ __forceinline__ explicit BlockScale(uint32_t big) {
        finite = big < 0x7f80u;
        const float m = __uint_as_float(big << 16);
        pre = m < 0x1p-100f ? 0x1p64f : 1.0f;
        r = finite && m > 0.0f ? 448.0f / (m * pre) : 0.0f;
    }
    __device__ __forceinline__ static float scale_of(uint32_t big) {
        const float m = __uint_as_float(big << 16);
        return big >= 0x7f80u ? __uint_as_float(0x7fffffffu) : m == 0.0f ? 1.0f : __fdiv_rn(m, 448.0f);
    }
    __device__ __forceinline__ float at_border(float x) const {   // the quotient with 13 fraction bits
        return __uint_as_float((__float_as_uint(x * pre * r) + 0x200u) & ~0x3ffu);
    }
    __device__ __forceinline__ uint32_t codes2(uint32_t x) const {
        const float2 v = make_float2(at_border(__uint_as_float(x << 16)), at_border(__uint_as_float(x & 0xffff0000u)));
        return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
    }
    __device__ __forceinline__ uint2 codes8(uint4 v) const {
        if (!finite) return make_uint2(0u, 0u);
        return make_uint2(codes2(v.x) | codes2(v.y) << 16, codes2(v.z) | codes2(v.w) << 16);
    }
};

// 1 x 128: half a warp per block, U blocks to a half warp.  333 x 2048 2.4 us (launch); 4096 x 2048 9.0, 24576 x 1408 28.5 us: 0.44 and 0.57
// of the measured copy rate.
template <int U>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const BlockArgs a) {
    grid_dependency();
    const int half = threadIdx.x >> 4, l = threadIdx.x & 15;
    const int64_t all = a.blocks * a.kb;
    const int64_t b0 = ((int64_t)blockIdx.x * U) * 16 + half;
    uint4 v[U];
    int64_t at[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t b = b0 + u * 16;
        const int64_t row = b / a.kb;
        const int col = (int)(b - row * a.kb) * 128 + l * 8;
        in[u] = b < all && col < a.cols;
        at[u] = row * a.cols + col;
        v[u] = in[u] ? load16(reinterpret_cast<const uint4 *>(a.w + at[u])) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t big = largest(v[u]);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
        const BlockScale s(big);
        if (in[u]) *reinterpret_cast<uint2 *>(a.q + at[u]) = s.codes8(v[u]);
        if (l == 0 && b0 + u * 16 < all) a.scale[b0 + u * 16] = BlockScale::scale_of(big);
    }
}

// 128 x 128: a thread block per block, which it holds in registers.  131072 x 1408 89 us, 0.96 of the measured copy rate.
__global__ void __launch_bounds__(256) quantize_squares_kernel(const BlockArgs a) {
    __shared__ uint32_t part[8];
    grid_dependency();
    const int row_blocks = a.rows / 128 + (a.rows % 128 != 0);   // (rows + 127 may not fit)
    const int64_t rb = blockIdx.x / a.kb;
    const int col = (int)(blockIdx.x - rb * a.kb) * 128 + (threadIdx.x & 15) * 8;
    const int64_t matrix = rb / row_blocks;
    const int row0 = (int)(rb - matrix * row_blocks) * 128 + (threadIdx.x >> 4);
    const int64_t base = (matrix * a.rows + row0) * a.cols + col;
    uint4 v[8];
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = col < a.cols && row0 + 16 * i < a.rows ? load16(reinterpret_cast<const uint4 *>(a.w + base + (int64_t)(16 * i) * a.cols))
                                                      : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, largest(v[i]));
    big = __reduce_max_sync(0xffffffffu, big);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = big;
    __syncthreads();
    big = part[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) big = max(big, part[w]);
    const BlockScale s(big);
    if (threadIdx.x == 0) a.scale[blockIdx.x] = BlockScale::scale_of(big);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col < a.cols && row0 + 16 * i < a.rows) *reinterpret_cast<uint2 *>(a.q + base + (int64_t)(16 * i) * a.cols) = s.codes8(v[i]);
}

}  // namespace

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_quantize_e4m3_blocks(const spice_bf16 *w, int64_t count, int64_t rows, int32_t cols, int32_t block_rows,
                                                   uint8_t *q, float *scale, void *stream) {
    Range range_("spice_quantize_e4m3_blocks");
    if (count < 0 || rows < 0 || cols < 8 || cols % 8 || (block_rows != 1 && block_rows != 128)) return SPICE_ERR_INVALID_ARG;
    if (cols > (1 << 24) || rows > 0x7fffffffLL || count > 0x7fffffffLL) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (count == 0 || rows == 0) return SPICE_OK;
    const int kb = (cols + 127) / 128;
    const int64_t row_blocks = block_rows == 1 ? rows : (rows + 127) / 128;
    if (row_blocks * count > (0x7fffffffLL * 16) / kb || (block_rows == 128 && row_blocks * count * kb > 0x7fffffffLL))
        return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (!w || !q || !scale || !aligned16(w) || (reinterpret_cast<uintptr_t>(q) & 7u) || (reinterpret_cast<uintptr_t>(scale) & 3u))
        return SPICE_ERR_INVALID_ARG;
    const BlockArgs a{reinterpret_cast<const __nv_bfloat16 *>(w), q, scale, row_blocks * count, (int32_t)rows, cols, kb};
    const int64_t blocks = a.blocks * kb;
    const int sms = current_device_sms();
    if (sms <= 0) return SPICE_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    bool ok;
    if (block_rows == 128) ok = launch_early(quantize_squares_kernel, dim3((unsigned)blocks), 256, 0, st, 1, a);
    else if (blocks < 16 * 4 * sms) ok = launch_early(quantize_rows_kernel<1>, dim3((unsigned)((blocks + 15) / 16)), 256, 0, st, 1, a);
    else ok = launch_early(quantize_rows_kernel<4>, dim3((unsigned)((blocks + 63) / 64)), 256, 0, st, 1, a);
    return ok ? SPICE_OK : SPICE_ERR_CUDA;
}
