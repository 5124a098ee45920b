// Rows in 8-bit integers: the residual addition with its root-mean-square norm (the step between two layers of the
// stack), and the quantiser of bf16 rows (weights once, SwiGLU activations every step).
//
//   s = bf16(x + delta), x <- s;   p_j = s_j * w_j,   r = 1 / sqrt(mean_j s_j^2 + eps),   h_j = bf16(p_j * r)
//   m = max_j |p_j|;   q_j = 127 p_j / m to the nearest integer, ties to even;   scale = m * r / 127
//
// (the quantiser: p = w, r = 1, no h).  r cancels out of q, and p is a product of two bf16 values, exact in fp32, so the
// codes are a function of exactly known numbers.  They are rounded exactly: where the fp32 quotient lies within its error
// of a border k + 1/2, 254 |p_j| and (2k + 1) m are compared, both exact in fp32 once m is scaled into [1, 2)
// (16 + 8 and 8 + 16 significant bits).  No implementation that keeps the definition can differ by a step.
//
// Both are bound by the bytes that cross HBM (9 per element of a bf16 step with both outputs, 3 for the quantiser): every
// row is read once, held in registers as the packed bf16 pairs it is stored as, and written once.
#include <type_traits>

#include "entry.cuh"
#include "spice_internal.cuh"

namespace spice {

namespace {

enum { DELTA_NONE = 0, DELTA_BF16 = 1, DELTA_F32 = 2, NO_NORM = 3 };

struct RowArgs {
    __nv_bfloat16 *x;             // [T, d] residual stream, in/out (NO_NORM: the rows, only read)
    const __nv_bfloat16 *delta;   // [T, d] DELTA_BF16
    const float *delta_f32;       // [T, d] DELTA_F32
    const __nv_bfloat16 *weight;  // [d]
    __nv_bfloat16 *h;             // [T, d] or null
    int8_t *q;                    // [T, d] or null
    float *scale;                 // [T], with q
    int d;
    float eps;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&b);
}

// Normaliser of one row's codes: multiplying by f (a power of two) brings the largest magnitude into [1, 2).
struct CodeScale {
    float f, inv, mn;
    __device__ __forceinline__ explicit CodeScale(float m) {
        const int e = (int)(__float_as_uint(m) >> 23);               // biased exponent of m >= 0
        f = __uint_as_float((uint32_t)min(max(254 - e, 1), 253) << 23);   // 2^(127 - e): at most 2^126
        mn = m * f;
        inv = m > 0.0f ? 127.0f / mn : 0.0f;
    }
};

// nearest integer to 127 p / m, ties to even, exactly (see the top of the file).  The fp32 quotient is off by at most
// 127 * 2^-22.9 < 2e-5.
__device__ __forceinline__ int code_of(float p, const CodeScale &c) {
    const float pn = p * c.f;
    const float u = pn * c.inv;
    float k = rintf(u);
    if (fabsf(u - k) > 0.4999f) {
        const float a = floorf(fabsf(u));
        const float lhs = 254.0f * fabsf(pn), rhs = (2.0f * a + 1.0f) * c.mn;
        const float up = lhs > rhs || (lhs == rhs && ((int)a & 1)) ? 1.0f : 0.0f;
        k = copysignf(a + up, u);
    }
    return (int)k;
}

__device__ __forceinline__ float warp_sum_xor(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// One row per group of threads: a warp (WIDE = false, several rows per block) or the whole block.  A thread holds V
// vectors of 8 elements, `step` threads apart.
template <int V, int MODE, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : 256) rows_i8_kernel(const RowArgs a, const size_t rows) {
    __shared__ float sh_sum[32];
    __shared__ uint32_t sh_max[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nw = blockDim.x >> 5;
    const size_t row = WIDE ? blockIdx.x : (size_t)blockIdx.x * nw + warp;
    if (!WIDE && row >= rows) return;
    const int i0 = WIDE ? threadIdx.x : lane, step = WIDE ? blockDim.x : 32;
    const int nv = a.d >> 3;
    const size_t base = row * (size_t)a.d;

    uint4 xs[V], dl[MODE == DELTA_BF16 ? V : 1], wt[MODE != NO_NORM ? V : 1];
    float4 df[MODE == DELTA_F32 ? 2 * V : 1];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = i0 + v * step;
        const bool in = i < nv;
        xs[v] = in ? *reinterpret_cast<const uint4 *>(a.x + base + (size_t)i * 8) : make_uint4(0, 0, 0, 0);
        if (MODE == DELTA_BF16)
            dl[v] = in ? *reinterpret_cast<const uint4 *>(a.delta + base + (size_t)i * 8) : make_uint4(0, 0, 0, 0);
        if (MODE == DELTA_F32) {
            const float4 *src = reinterpret_cast<const float4 *>(a.delta_f32 + base + (size_t)i * 8);
            df[2 * v] = in ? src[0] : make_float4(0.f, 0.f, 0.f, 0.f);
            df[2 * v + 1] = in ? src[1] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        if (MODE != NO_NORM) wt[v] = in ? *reinterpret_cast<const uint4 *>(a.weight + (size_t)i * 8) : make_uint4(0, 0, 0, 0);
    }

    float sum = 0.0f;
    uint32_t big = 0;   // bits of |p|: magnitudes order like integers, infinities and NaN on top
#pragma unroll
    for (int v = 0; v < V; ++v) {
        uint32_t *x = reinterpret_cast<uint32_t *>(&xs[v]);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&wt[MODE != NO_NORM ? v : 0]);
        const uint32_t *d16 = reinterpret_cast<const uint32_t *>(&dl[MODE == DELTA_BF16 ? v : 0]);
        const float *d32 = reinterpret_cast<const float *>(&df[MODE == DELTA_F32 ? 2 * v : 0]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (MODE == DELTA_BF16) x[j] = pack_bf16(bf_lo(x[j]) + bf_lo(d16[j]), bf_hi(x[j]) + bf_hi(d16[j]));
            if (MODE == DELTA_F32) x[j] = pack_bf16(bf_lo(x[j]) + d32[2 * j], bf_hi(x[j]) + d32[2 * j + 1]);
            const float lo = bf_lo(x[j]), hi = bf_hi(x[j]);
            if (MODE == NO_NORM) {
                big = max(big, max(__float_as_uint(lo) & 0x7fffffffu, __float_as_uint(hi) & 0x7fffffffu));
            } else {
                sum = fmaf(lo, lo, sum);
                sum = fmaf(hi, hi, sum);
                big = max(big, max(__float_as_uint(lo * bf_lo(w[j])) & 0x7fffffffu, __float_as_uint(hi * bf_hi(w[j])) & 0x7fffffffu));
            }
        }
        const int i = i0 + v * step;
        if ((MODE == DELTA_BF16 || MODE == DELTA_F32) && i < nv) *reinterpret_cast<uint4 *>(a.x + base + (size_t)i * 8) = xs[v];
    }
    big = __reduce_max_sync(0xffffffffu, big);
    if (MODE != NO_NORM) sum = warp_sum_xor(sum);
    if (WIDE) {
        if (lane == 0) {
            sh_sum[warp] = sum;
            sh_max[warp] = big;
        }
        __syncthreads();
        big = __reduce_max_sync(0xffffffffu, lane < nw ? sh_max[lane] : 0u);
        if (MODE != NO_NORM) sum = warp_sum_xor(lane < nw ? sh_sum[lane] : 0.0f);
    }
    const bool finite = big < 0x7f800000u;
    float r = 1.0f;
    if (MODE != NO_NORM) {
        const float mean = sum / (float)a.d + a.eps;
        r = 1.0f / sqrtf(mean);
        if (finite && !(mean >= 0x1p-60f && mean < INFINITY)) {   // (the same for the whole row)
            // squares at the ends of fp32's range: once more, of scaled values
            const float S = mean < 1.0f ? 0x1p64f : 0x1p-100f;
            float s2 = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t *x = reinterpret_cast<const uint32_t *>(&xs[v]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float lo = bf_lo(x[j]) * S, hi = bf_hi(x[j]) * S;
                    s2 = fmaf(lo, lo, s2);
                    s2 = fmaf(hi, hi, s2);
                }
            }
            s2 = warp_sum_xor(s2);
            if (WIDE) {
                __syncthreads();
                if (lane == 0) sh_sum[warp] = s2;
                __syncthreads();
                s2 = warp_sum_xor(lane < nw ? sh_sum[lane] : 0.0f);
            }
            r = S / sqrtf(s2 / (float)a.d + a.eps * S * S);
        }
    }
    const float m = __uint_as_float(big);
    const bool codes = finite && (r < INFINITY || m == 0.0f);
    if (a.q && i0 == 0) {
        constexpr float C = 1.0f / 127.0f;
        a.scale[row] = !codes ? __uint_as_float(0x7fffffffu) : m == 0.0f ? 1.0f : m > 1.0f ? (m * C) * r : m * (r * C);
    }
    const CodeScale cs(finite ? m : 0.0f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = i0 + v * step;
        if (i >= nv) break;
        const uint32_t *x = reinterpret_cast<const uint32_t *>(&xs[v]);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&wt[MODE != NO_NORM ? v : 0]);
        uint32_t hv[4], qv[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float lo = bf_lo(x[j]), hi = bf_hi(x[j]);
            if (MODE != NO_NORM) {
                lo *= bf_lo(w[j]);
                hi *= bf_hi(w[j]);
                hv[j] = pack_bf16(lo * r, hi * r);
            }
            if (a.q && codes)
                qv[j >> 1] |= ((uint32_t)(code_of(lo, cs) & 0xff) | (uint32_t)(code_of(hi, cs) & 0xff) << 8) << (16 * (j & 1));
        }
        if (MODE != NO_NORM && a.h) *reinterpret_cast<uint4 *>(a.h + base + (size_t)i * 8) = make_uint4(hv[0], hv[1], hv[2], hv[3]);
        if (a.q) *reinterpret_cast<uint2 *>(a.q + base + (size_t)i * 8) = make_uint2(qv[0], qv[1]);
    }
}

constexpr int MAX_COLS = 32768;   // 512 threads x 8 vectors x 8 elements: what a block holds in registers

template <int MODE>
spice_status launch_rows(const RowArgs &a, size_t rows, cudaStream_t st) {
    const int nv = a.d >> 3;
    auto wide = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int threads = ((nv + V - 1) / V + 31) & ~31;
        rows_i8_kernel<V, MODE, true><<<(unsigned)rows, threads, 0, st>>>(a, rows);
    };
    auto narrow = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int wpb = rows < 8 * 296 ? 4 : 8;
        rows_i8_kernel<V, MODE, false><<<(unsigned)((rows + wpb - 1) / wpb), wpb * 32, 0, st>>>(a, rows);
    };
    using std::integral_constant;
    if (nv <= 32) narrow(integral_constant<int, 1>{});
    else if (nv <= 64) narrow(integral_constant<int, 2>{});
    else if (nv <= 512) wide(integral_constant<int, 1>{});
    else if (nv <= 1024) wide(integral_constant<int, 2>{});
    else if (nv <= 2048) wide(integral_constant<int, 4>{});
    else wide(integral_constant<int, 8>{});
    return cudaGetLastError() == cudaSuccess ? SPICE_OK : SPICE_ERR_CUDA;
}

}  // namespace

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_residual_rmsnorm(spice_bf16 *x_resid, const spice_bf16 *delta, const float *delta_f32,
                                               const spice_bf16 *weight, float eps, int32_t T, int32_t d, spice_bf16 *h,
                                               int8_t *q, float *scale, void *stream) {
    Range range_("spice_residual_rmsnorm");
    if (T < 0 || d < 8 || d % 8 || !(eps >= 0.0f)) return SPICE_ERR_INVALID_ARG;
    if (d > MAX_COLS) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    if ((delta && delta_f32) || (!h && !q) || (q && !scale)) return SPICE_ERR_INVALID_ARG;
    if (!x_resid || !weight || !aligned16(x_resid) || !aligned16(delta) || !aligned16(delta_f32) || !aligned16(weight) ||
        !aligned16(h) || (reinterpret_cast<uintptr_t>(q) & 7u) || (reinterpret_cast<uintptr_t>(scale) & 3u))
        return SPICE_ERR_INVALID_ARG;
    const RowArgs a{reinterpret_cast<__nv_bfloat16 *>(x_resid), reinterpret_cast<const __nv_bfloat16 *>(delta), delta_f32,
                    reinterpret_cast<const __nv_bfloat16 *>(weight), reinterpret_cast<__nv_bfloat16 *>(h), q, scale, d, eps};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (delta) return launch_rows<DELTA_BF16>(a, (size_t)T, st);
    if (delta_f32) return launch_rows<DELTA_F32>(a, (size_t)T, st);
    return launch_rows<DELTA_NONE>(a, (size_t)T, st);
}

extern "C" spice_status spice_quantize_i8_rows(const spice_bf16 *w, int64_t rows, int32_t cols, int8_t *q, float *scale,
                                               void *stream) {
    Range range_("spice_quantize_i8_rows");
    if (rows < 0 || cols < 8 || cols % 8) return SPICE_ERR_INVALID_ARG;
    if (cols > MAX_COLS || rows > 0x7fffffffLL) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (rows == 0) return SPICE_OK;
    if (!w || !q || !scale || !aligned16(w) || (reinterpret_cast<uintptr_t>(q) & 7u) || (reinterpret_cast<uintptr_t>(scale) & 3u))
        return SPICE_ERR_INVALID_ARG;
    // (the kernel only reads x in this mode)
    const RowArgs a{const_cast<__nv_bfloat16 *>(reinterpret_cast<const __nv_bfloat16 *>(w)), nullptr, nullptr, nullptr, nullptr,
                    q, scale, cols, 0.0f};
    return launch_rows<NO_NORM>(a, (size_t)rows, static_cast<cudaStream_t>(stream));
}
