// Products of 8-bit floating-point rows with a scale for each block of 128, dense or over rows sorted by expert:
//
//   y[t, j] = sum_b xs[t,b] ws[j/128, b] sum_{i in block b} x[t,i] w[j,i]            (bf16, fp32, or added to fp32)
//   SwiGLU:   g, u = the products with the gate and the up rows;  a = g / (1 + e^-g) u;  codes and scales of a in blocks of 128
//
// with the weights of group g for the rows offset[g] .. offset[g+1].  The inner sums are 128 products of E4M3 values, exact
// in the tensor cores' operands and added in their fp32 accumulators; every block's sum is multiplied by its two scales and
// added in fp32 registers, so no scale is rounded into an operand and long reductions are sums of fp32 sums.
//
// Two kernels.  Few rows a group: every weight byte is used for few products and the call is bound by streaming the weights:
// they go from global memory straight into the registers of warp-wide products.  Otherwise pairs of CTAs (cta_group::2) work on
// tiles of 256 weight rows x up to 256 tokens, persistent.  The weights are the M operand, so that the tokens' side of a tile is as
// wide as the group's rows need (a multiple of 32): groups are ragged, and a tile of 256 tokens would be padding for a third.
#include <cuda_fp8.h>

#include <algorithm>
#include <mutex>

#include "entry.cuh"
#include "spice_internal.cuh"
#include "tc_device.cuh"

namespace spice {

namespace {

using namespace tcdev;

constexpr int BK = 128;                 // bytes = elements of the reduction per block of scales and pipeline stage
constexpr int MAX_GROUPS = 1024;

struct GemmE4m3Args {
    const float *xs, *ws;    // [T, kb], [G, row blocks, kb]
    const int32_t *offset;   // [G + 1], or null: one group of all T rows
    void *y;                 // [T, n] (SwiGLU: codes [T, n])
    float *ys;               // SwiGLU: [T, n / 128]
    int32_t T, n, k, G;      // n: columns of y
    int32_t kb;              // blocks of the reduction
    int32_t out;             // SPICE_OUT_*
    int32_t *status;         // optional
    uint32_t wait_limit;     // polls after which a wait inside a kernel gives up
    int32_t n_tiles;         // tiles along n
};

// (fast exponential and quotient: a few 2^-23 for |g| of some units)
__device__ __forceinline__ float silu_times(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ float load_f32(const float *p) {   // (not as constant: the kernel may be set up early)
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ int32_t load_s32(const int32_t *p) {
    int32_t v;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pair2(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float low(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }

// The scale of a block of SwiGLU outputs with largest magnitude m, and what its values are multiplied with.  A block with a
// value that is not finite: scale NaN, codes 0.  A block below 2^-100 (448 / m nears the end of fp32) is taken for zeros.
struct OutScale {
    float scale, r;
    __device__ __forceinline__ explicit OutScale(float m) {
        const bool finite = m < __uint_as_float(0x7f800000u), live = finite && m >= 0x1p-100f;
        scale = live ? m * (1.0f / 448.0f) : finite ? 1.0f : __uint_as_float(0x7fffffffu);
        r = live ? 448.0f / m : 0.0f;
    }
};
__device__ __forceinline__ uint32_t code2(float a, float b, float r) {
    return r == 0.0f ? 0u : __nv_cvt_float2_to_fp8x2(make_float2(a * r, b * r), __NV_SATFINITE, __NV_E4M3);
}
// the larger magnitude; NaN if there is one
__device__ __forceinline__ float max_magnitude(float m, float a) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(a)));
    return r;
}

__device__ __forceinline__ void store1(const GemmE4m3Args &g, size_t at, float v) {
    if (g.out == SPICE_OUT_BF16) static_cast<__nv_bfloat16 *>(g.y)[at] = __float2bfloat16_rn(v);
    else if (g.out == SPICE_OUT_F32) static_cast<float *>(g.y)[at] = v;
    else static_cast<float *>(g.y)[at] += v;
}

// ------------------------------------------------------------------------------------------------ few rows a group
// A block multiplies 16 weight rows (SwiGLU: 16 gate rows and their up rows) with the rows of one group, eight or sixteen at a
// time; its warps share the blocks of the reduction.  Both operands are read in pieces of 16 bytes, so the order of the reduction
// inside a 64-byte piece is the same for both and does not matter.  SwiGLU: eight blocks of a cluster hold the 128 columns of an
// output block and exchange their largest values.
constexpr int FEW_WARPS = 8, FEW_CLUSTER = 8;

__device__ __forceinline__ int4 load_once(const int4 *p) {
    int4 v;
    asm volatile("ld.global.cs.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int4 load_again(const int4 *p) {
    int4 v;
    asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], int a0, int a1, int a2, int a3, int b0, int b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The slot-th group that has rows: its number, or -1; groups whose offsets are not in order or out of range have none.
__device__ __forceinline__ int find_group(const GemmE4m3Args &g, int slot, int32_t *off, int &begin, int &rows) {
    for (int i = threadIdx.x; i <= g.G; i += blockDim.x) off[i] = load_s32(g.offset + i);
    __syncthreads();
    auto bad = [&](int i) { return off[i] < 0 || off[i + 1] < off[i] || off[i + 1] > g.T; };
    if (blockIdx.x == 0 && slot == 0 && g.status)
        for (int i = threadIdx.x; i < g.G; i += blockDim.x)
            if (bad(i)) atomicMax(g.status, (int)SPICE_ERR_BAD_TABLE);
    const int lane = threadIdx.x & 31;
    int seen = 0;
    for (int base = 0; base < g.G; base += 32) {
        const int i = base + lane;
        uint32_t mask = __ballot_sync(0xffffffffu, i < g.G && !bad(i) && off[i + 1] > off[i]);
        const int here = __popc(mask);
        if (seen + here > slot) {
            for (int s = slot - seen; s > 0; --s) mask &= mask - 1;
            const int found = base + __ffs(mask) - 1;
            begin = off[found];
            rows = off[found + 1] - begin;
            return found;
        }
        seen += here;
    }
    return -1;
}

template <int NT, bool SWIGLU>
__global__ void __launch_bounds__(FEW_WARPS * 32) gemm_e4m3_few_kernel(const uint8_t *x, const uint8_t *w, const GemmE4m3Args g) {
    constexpr int RT = SWIGLU ? 2 : 1, UN = NT * RT > 2 ? 1 : 2;
    __shared__ float red[FEW_WARPS][NT * 8][RT * 16 + 4];   // (padded: the 8 rows of a warp's store fall into different banks)
    __shared__ int32_t off[MAX_GROUPS + 1];
    __shared__ float peak[NT * 8];                          // SwiGLU: largest magnitude of each token's 16 columns
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gq = lane >> 2, c = lane & 3;
    const int n0 = blockIdx.x * 16;
    grid_dependency();
    int group = 0, begin = 0, rows = g.T;
    if (g.offset) {
        group = find_group(g, blockIdx.y, off, begin, rows);
        if (group < 0) return;                              // (the same for every block of a cluster)
    }
    const int w_rows = SWIGLU ? 2 * g.n : g.n, row_blocks = (w_rows + 127) / 128;
    const int4 *wr[RT][2];
    const float *ws[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int first = r * g.n + n0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = first + gq + (n0 + 8 * h < g.n ? 8 * h : 0);   // (n is a multiple of 8)
            wr[r][h] = reinterpret_cast<const int4 *>(w + ((size_t)group * w_rows + row) * g.k);
        }
        ws[r] = g.ws + ((size_t)group * row_blocks + first / 128) * g.kb;
    }
    const int nv = g.k >> 4;
    for (int t0 = 0; t0 < rows; t0 += NT * 8) {
        const int m = min(rows - t0, NT * 8), row0 = begin + t0;
        const int4 *x4 = reinterpret_cast<const int4 *>(x) + (size_t)row0 * nv;
        const float *xs = g.xs + (size_t)row0 * g.kb;
        float acc[RT][NT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][i][j] = 0.0f;
        const int4 zero = make_int4(0, 0, 0, 0);
        for (int b0 = warp; b0 < g.kb; b0 += FEW_WARPS * UN) {
            int4 a[UN][RT][2][2], bx[UN][2][NT];
            float sx[UN][NT][2], sw[UN][RT];
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const int b = b0 + u * FEW_WARPS;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int v = b * 8 + p * 4 + c;
                    const bool in = b < g.kb && v < nv;
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h) a[u][r][p][h] = in ? load_once(wr[r][h] + v) : zero;
                }
            }
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const int b = b0 + u * FEW_WARPS;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int v = b * 8 + p * 4 + c;
#pragma unroll
                    for (int i = 0; i < NT; ++i)
                        bx[u][p][i] = b < g.kb && v < nv && i * 8 + gq < m ? load_again(x4 + (size_t)(i * 8 + gq) * nv + v) : zero;
                }
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int t = i * 8 + 2 * c + j;
                        sx[u][i][j] = b < g.kb && t < m ? load_f32(xs + (size_t)t * g.kb + b) : 0.0f;
                    }
#pragma unroll
                for (int r = 0; r < RT; ++r) sw[u][r] = b < g.kb ? load_f32(ws[r] + b) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < UN; ++u)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const int4 a0 = a[u][r][p][0], a1 = a[u][r][p][1], bb = bx[u][p][i];
                            mma_e4m3(d, a0.x, a1.x, a0.y, a1.y, bb.x, bb.y);
                            mma_e4m3(d, a0.z, a1.z, a0.w, a1.w, bb.z, bb.w);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[r][i][j] = fmaf(d[j], sx[u][i][j & 1] * sw[u][r], acc[r][i][j]);
                    }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < NT; ++i) {   // rows gq, gq + 8 x tokens 2c, 2c + 1
                red[warp][i * 8 + 2 * c][r * 16 + gq] = acc[r][i][0];
                red[warp][i * 8 + 2 * c + 1][r * 16 + gq] = acc[r][i][1];
                red[warp][i * 8 + 2 * c][r * 16 + gq + 8] = acc[r][i][2];
                red[warp][i * 8 + 2 * c + 1][r * 16 + gq + 8] = acc[r][i][3];
            }
        __syncthreads();
        constexpr int ITEMS = NT * 8 * 16;   // one per thread at most
        static_assert(ITEMS <= FEW_WARPS * 32, "an output per thread");
        const int t = threadIdx.x / 16, r = threadIdx.x % 16;
        float v = 0.0f, u = 0.0f;
        if (threadIdx.x < ITEMS) {
#pragma unroll
            for (int q = 0; q < FEW_WARPS; ++q) {
                v += red[q][t][r];
                if (SWIGLU) u += red[q][t][16 + r];
            }
        }
        if constexpr (!SWIGLU) {
            if (threadIdx.x < ITEMS && t < m && n0 + r < g.n) store1(g, (size_t)(row0 + t) * g.n + n0 + r, v);
            __syncthreads();   // the sums have been read
        } else {
            v = silu_times(v, u);
            float big = fabsf(v);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) big = max_magnitude(big, __shfl_xor_sync(0xffffffffu, big, o));
            if (threadIdx.x < ITEMS && r == 0) peak[t] = big;
            cluster_sync();
            if (threadIdx.x < ITEMS) {
                const uint32_t at = smem_u32(&peak[t]);
#pragma unroll
                for (uint32_t p = 0; p < FEW_CLUSTER; ++p) {
                    float o;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o) : "r"(map_to_cta(at, p)));
                    big = max_magnitude(big, o);
                }
                const OutScale s(big);
                if (t < m) {
                    static_cast<uint8_t *>(g.y)[(size_t)(row0 + t) * g.n + n0 + r] = (uint8_t)code2(v, 0.0f, s.r);
                    if (r == 0 && n0 % 128 == 0) g.ys[(size_t)(row0 + t) * (g.n / 128) + n0 / 128] = s.scale;
                }
            }
            cluster_sync();    // nobody writes its next values, or leaves, while a peer reads
        }
    }
}

// ------------------------------------------------------------------------------------------------ more rows
constexpr int PR_THREADS = 384, PR_STAGES = 6, PR_EPI_WARPS = 8;
constexpr int PR_TILE = 256;                      // weight rows of a pair's tile (128 per CTA), and its most tokens
constexpr int PR_W_BYTES = 128 * BK, PR_X_BYTES = 128 * BK, PR_STAGE_BYTES = PR_W_BYTES + PR_X_BYTES;
constexpr int PR_BATCH = 4;                       // blocks of the reduction whose scales are staged at a time
constexpr int PR_GROUP_M = 16;                    // token tiles that share a sweep over the weight tiles
constexpr int PR_PITCH = 80;                      // 64 B of a token's outputs + 16: 16-byte accesses do not collide
constexpr int PR_F32_PITCH = 144;                 // the same for 128 B
constexpr int PR_STG_WARP = 2048;                 // a warp's transposition buffers: 8 tokens x 32 columns, bf16 twice
static_assert(2 * 8 * PR_PITCH <= PR_STG_WARP && 8 * PR_F32_PITCH <= PR_STG_WARP, "they fit");
// The sums of a tile take 128 registers of each epilogue thread: the four warps that copy and multiply give theirs up.
constexpr int PR_REGS_HELPERS = 40, PR_REGS_EPILOGUE = 232;
static_assert(PR_REGS_HELPERS + 2 * PR_REGS_EPILOGUE <= 3 * (65536 / PR_THREADS / 8 * 8), "what the block is launched with");

struct PairShared {
    alignas(16) float xs[2][PR_BATCH][PR_TILE];   // token scales (product: times the weights' scale); the buffer that is not in
                                                  // use also takes the largest magnitudes of a token's columns (SwiGLU)
    alignas(16) unsigned char stg[PR_EPI_WARPS * PR_STG_WARP];   // transposition buffers; SwiGLU: [256 tokens][64 codes]
    float other[2][PR_TILE];                      // SwiGLU: the largest magnitudes of the other CTA's columns, which it writes here
    int32_t first[MAX_GROUPS + 1];                // tiles before each group
    alignas(8) unsigned long long full[PR_STAGES], empty[PR_STAGES], tmem_full[2], tmem_empty[2], mma_drain, peer[2];
    uint32_t tmem_base;
    int abort_flag;
};
constexpr size_t PR_SMEM_BYTES = sizeof(PairShared) + (size_t)PR_STAGES * PR_STAGE_BYTES + 1024;
static_assert(PR_SMEM_BYTES <= 232448, "what a block can have");
static_assert(PR_TILE * 64 <= PR_EPI_WARPS * PR_STG_WARP && 4 <= PR_BATCH, "codes and largest magnitudes fit");

struct Tile {
    int group, t0, cols, nt;   // first token, tokens, weight tile
};

// tokens of a tile as the products of a pair take them
__device__ __forceinline__ int padded(int tokens) { return (tokens + 31) & ~31; }

// Tiles are numbered group by group; within a group sweeps of up to PR_GROUP_M token tiles, the token tile fastest, so that
// pairs working at the same time share both operands in L2.  A group's rows are spread evenly over as few token tiles as there
// can be.  The group only moves forward.
__device__ __forceinline__ Tile find_tile(const PairShared &sh, const GemmE4m3Args &g, int tile, int &group) {
    while (tile >= sh.first[group + 1]) ++group;
    const int begin = g.offset ? load_s32(g.offset + group) : 0, m = (g.offset ? load_s32(g.offset + group + 1) : g.T) - begin;
    const int in = tile - sh.first[group];
    const int tt = (m + PR_TILE - 1) / PR_TILE, width = padded((m + tt - 1) / tt);
    const int per_sweep = PR_GROUP_M * g.n_tiles;
    const int sweep = in / per_sweep, mt0 = sweep * PR_GROUP_M, left = min(PR_GROUP_M, tt - mt0), r = in - sweep * per_sweep;
    const int mt = mt0 + r % left;
    return Tile{group, begin + mt * width, min(width, m - mt * width), r / left};
}

template <bool SWIGLU>
__global__ void __launch_bounds__(PR_THREADS, 1)
    gemm_e4m3_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x64,
                          const __grid_constant__ CUtensorMap map_x32, const __grid_constant__ CUtensorMap map_x16, const GemmE4m3Args g) {
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    PairShared &sh = *reinterpret_cast<PairShared *>(ring + PR_STAGES * PR_STAGE_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    volatile int *abort_flag = &sh.abort_flag;

    if (threadIdx.x == 0) {
        for (int s = 0; s < PR_STAGES; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);    // used in the even CTA: both CTAs' copies report there
            mbar_init(smem_u32(&sh.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh.tmem_full[b]), 1);
            mbar_init(smem_u32(&sh.tmem_empty[b]), 2 * PR_EPI_WARPS);   // used in the even CTA: the epilogue warps of both
            mbar_init(smem_u32(&sh.peer[b]), PR_EPI_WARPS);             // the other CTA's epilogue warps
        }
        mbar_init(smem_u32(&sh.mma_drain), 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {   // TMEM: all 512 columns (two 256-column accumulators), in both CTAs
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
    }
    grid_dependency();
    if (warp == 2) {   // tiles before each group; a group whose offsets are not in order or out of range has none
        int carry = 0;
        for (int base = 0; base < g.G; base += 32) {
            const int i = base + lane;
            int b = 0, e = g.T, tiles = 0;
            if (i < g.G && g.offset) {
                b = load_s32(g.offset + i);
                e = load_s32(g.offset + i + 1);
            }
            if (i < g.G) {
                if (b < 0 || e < b || e > g.T) {
                    if (blockIdx.x == 0 && g.status) atomicMax(g.status, (int)SPICE_ERR_BAD_TABLE);
                } else {
                    tiles = (e - b + PR_TILE - 1) / PR_TILE * g.n_tiles;
                }
            }
            int incl = tiles;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (i < g.G) sh.first[i] = carry + incl - tiles;
            carry += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) sh.first[g.G] = carry;
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // both CTAs' barriers exist before either signals the other's
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    const int n_tiles = sh.first[g.G];
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int row_blocks = ((SWIGLU ? 2 * g.n : g.n) + 127) / 128;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_HELPERS));
        if (warp == 0 && lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            int group = 0;
            for (int tile = pair; tile < n_tiles && ok; tile += pairs) {
                const Tile t = find_tile(sh, g, tile, group);
                const int half = padded(t.cols) / 2, x_row = t.t0 + (int)rank * half;
                for (int kb = 0; kb < g.kb; ++kb, ++it) {
                    const int s = it % PR_STAGES;
                    if (!mbar_wait(smem_u32(&sh.empty[s]), ((it / PR_STAGES) & 1) ^ 1, abort_flag, g.wait_limit)) { ok = false; break; }
                    const uint32_t full = map_to_cta(smem_u32(&sh.full[s]), 0);
                    const uint32_t dst = smem_u32(ring + s * PR_STAGE_BYTES);
                    if (rank == 0) mbar_expect_tx(smem_u32(&sh.full[s]), 2 * (PR_W_BYTES + half * BK));
                    if (SWIGLU) tma_load_5d_pair(dst, &map_w, kb * BK, 0, 0, 2 * t.group, t.nt * 8 + (int)rank * 4, full);
                    else tma_load_2d_pair(dst, &map_w, kb * BK, t.group * g.n + t.nt * PR_TILE + (int)rank * 128, full);
                    uint32_t to = dst + PR_W_BYTES;
                    int row = x_row;
                    auto rows = [&](const CUtensorMap *map, int n) {
                        tma_load_2d_pair(to, map, kb * BK, row, full);
                        to += n * BK;
                        row += n;
                    };
                    if (half & 128) rows(&map_x64, 64);
                    if (half & (128 | 64)) rows(&map_x64, 64);
                    if (half & 32) rows(&map_x32, 32);
                    if (half & 16) rows(&map_x16, 16);
                }
            }
            // a CTA ends when the stages it filled have been read by the MMAs: nothing of it is in flight then, neither a
            // copy nor a release of a stage (also after an abort, within the limit: copies have long landed by then)
            for (uint32_t j = (it > PR_STAGES ? it - PR_STAGES : 0); j < it; ++j)
                if (!mbar_drain(smem_u32(&sh.empty[j % PR_STAGES]), (j / PR_STAGES) & 1)) {
                    *abort_flag = 1;
                    break;
                }
        } else if (warp == 1 && rank == 0 && lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            int group = 0;
            for (int tile = pair; tile < n_tiles && ok; tile += pairs) {
                const Tile t = find_tile(sh, g, tile, group);
                const uint32_t idesc = make_idesc_e4m3(256, padded(t.cols));
                for (int kb = 0; kb < g.kb; ++kb, ++it) {
                    const int s = it % PR_STAGES, buf = it & 1;
                    if (!mbar_wait(smem_u32(&sh.tmem_empty[buf]), ((it >> 1) & 1) ^ 1, abort_flag, g.wait_limit)) { ok = false; break; }
                    if (!mbar_wait(smem_u32(&sh.full[s]), (it / PR_STAGES) & 1, abort_flag, g.wait_limit)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a0 = smem_u32(ring + s * PR_STAGE_BYTES);
                    const uint64_t da = make_desc(a0), db = make_desc(a0 + PR_W_BYTES);
#pragma unroll
                    for (int k = 0; k < BK / 32; ++k) tc_mma_f8_pair(tmem_base + buf * PR_TILE, da + 2 * k, db + 2 * k, idesc, k ? 1u : 0u);
                    tc_commit_pair(smem_u32(&sh.empty[s]), 3u);
                    tc_commit_pair(smem_u32(&sh.tmem_full[buf]), 3u);
                }
            }
            tc_commit_pair_local(smem_u32(&sh.mma_drain));
            if (!mbar_drain(smem_u32(&sh.mma_drain), 0)) *abort_flag = 1;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PR_REGS_EPILOGUE));
        // ---------------- epilogue: warp w reads TMEM lanes 32*(w%4) .. +31 = weight rows of this CTA's half of the tile; the two
        // warps of a quarter take half of the tokens each.  Sums are held in registers in the layout of warp-wide products: a
        // thread has two neighbouring tokens of every eight, so that it needs a quarter of the tokens' scales.
        const int q = warp & 3, h = warp >= 8 ? 1 : 0, e = threadIdx.x - 128;
        const int r4 = lane >> 2, c2 = 2 * (lane & 3);
        uint32_t it = 0, batch = 0, count = 0;   // blocks, batches of scales and tiles so far
        int group = 0;
        bool ok = true;   // after an expired wait a warp only keeps the others' barriers
        for (int tile = pair; tile < n_tiles; tile += pairs, ++count) {
            const Tile t = find_tile(sh, g, tile, group);
            const int cols = padded(t.cols), mine = cols / 2, col0 = h * mine;
            const int nb = SWIGLU ? t.nt : t.nt * 2 + (int)rank;    // block of weight rows
            const float *ws = g.ws + ((size_t)t.group * row_blocks + min(nb, row_blocks - 1)) * g.kb;
            const float *ws_up = SWIGLU ? ws + (size_t)(g.n / 128) * g.kb : ws;
            const float *xs = g.xs + (size_t)(t.t0 + min(e, t.cols - 1)) * g.kb;
            uint64_t acc[16][2][2];   // [eight tokens][16 rows][rows r4, r4 + 8]: two tokens
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i][0][0] = acc[i][0][1] = acc[i][1][0] = acc[i][1][1] = 0;
            float next[PR_BATCH], next_w[PR_BATCH];
            auto fetch = [&](int kb0) {
#pragma unroll
                for (int j = 0; j < PR_BATCH; ++j) {
                    next[j] = kb0 + j < g.kb ? load_f32(xs + kb0 + j) : 0.0f;
                    if (!SWIGLU) next_w[j] = kb0 + j < g.kb ? load_f32(ws + kb0 + j) : 0.0f;
                }
            };
            fetch(0);
            for (int kb0 = 0; kb0 < g.kb; kb0 += PR_BATCH, ++batch) {
                float (*stage)[PR_TILE] = sh.xs[batch & 1];
#pragma unroll
                for (int j = 0; j < PR_BATCH; ++j) stage[j][e] = SWIGLU ? next[j] : next[j] * next_w[j];
                fetch(kb0 + PR_BATCH);
                // (a warp that writes a buffer again has seen this barrier after the batch before: everyone has read it)
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const int last = min(PR_BATCH, g.kb - kb0);
                for (int j = 0; j < last; ++j, ++it) {
                    const int buf = it & 1;
                    uint64_t wg = 0, wu = 0;
                    if (SWIGLU) {
                        const float a = load_f32(ws + kb0 + j), b = load_f32(ws_up + kb0 + j);
                        wg = pair2(a, a);
                        wu = pair2(b, b);
                    }
                    if (ok && lane == 0) ok = mbar_wait(smem_u32(&sh.tmem_full[buf]), (it >> 1) & 1, abort_flag, g.wait_limit);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (!ok) continue;
                    tc_fence_after();
                    const uint32_t tm = tmem_base + buf * PR_TILE + col0 + ((uint32_t)(q * 32) << 16);
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        if (ch * 32 >= mine) break;
                        uint32_t v0[16], v1[16];
                        tc_ld_fragments(tm + ch * 32, v0);
                        tc_ld_fragments(tm + ch * 32 + (16u << 16), v1);
                        uint64_t s[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[i] = *reinterpret_cast<const uint64_t *>(&stage[j][(col0 + ch * 32 + i * 8 + c2) & (PR_TILE - 1)]);
                        tc_wait_ld();
                        if (ch * 32 + 32 >= mine) {   // the last columns are in registers: the buffer is free
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&sh.tmem_empty[buf]), 0));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint64_t sg = SWIGLU ? mul2(s[i], wg) : s[i], su = SWIGLU ? mul2(s[i], wu) : s[i];
                            uint64_t (&a)[2][2] = acc[ch * 4 + i];
                            a[0][0] = fma2(pair2(v0[4 * i], v0[4 * i + 1]), sg, a[0][0]);
                            a[0][1] = fma2(pair2(v0[4 * i + 2], v0[4 * i + 3]), sg, a[0][1]);
                            a[1][0] = fma2(pair2(v1[4 * i], v1[4 * i + 1]), su, a[1][0]);
                            a[1][1] = fma2(pair2(v1[4 * i + 2], v1[4 * i + 3]), su, a[1][1]);
                        }
                    }
                }
            }
            if constexpr (SWIGLU) {
                // rows 2 r4, 2 r4 + 1 of this quarter's 16 (the copy laid the weight rows out that way): activations into acc[.][0]
                const int b2 = count & 1;
                float (*peak)[PR_TILE] = sh.xs[batch & 1];   // (the last batch may still be read; everyone is past the one before)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i * 8 >= mine) break;
                    float big0 = 0.0f, big1 = 0.0f;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float a0 = silu_times(low(acc[i][0][r]), low(acc[i][1][r])), a1 = silu_times(high(acc[i][0][r]), high(acc[i][1][r]));
                        acc[i][0][r] = pair2(a0, a1);
                        big0 = max_magnitude(big0, a0);
                        big1 = max_magnitude(big1, a1);
                    }
#pragma unroll
                    for (int o = 4; o < 32; o *= 2) {
                        big0 = max_magnitude(big0, __shfl_xor_sync(0xffffffffu, big0, o));
                        big1 = max_magnitude(big1, __shfl_xor_sync(0xffffffffu, big1, o));
                    }
                    if (lane < 4) *reinterpret_cast<float2 *>(&peak[q][col0 + i * 8 + c2]) = make_float2(big0, big1);
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                // this CTA's largest values, and the other's (two buffers: neither CTA can be more than a tile ahead)
                float own = 0.0f;
                if (e < cols) {
#pragma unroll
                    for (int p = 0; p < 4; ++p) own = max_magnitude(own, peak[p][e]);
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(smem_u32(&sh.other[b2][e]), rank ^ 1u)), "f"(own) : "memory");
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_cluster(map_to_cta(smem_u32(&sh.peer[b2]), rank ^ 1u));
                    if (ok) ok = mbar_wait_cluster(smem_u32(&sh.peer[b2]), (count >> 1) & 1, abort_flag, g.wait_limit);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                __syncwarp();
                if (e < cols) {
                    const OutScale s(max_magnitude(own, *(volatile float *)&sh.other[b2][e]));
                    peak[0][e] = s.r;   // (only this thread looked at its token's column)
                    if (ok && rank == 0 && e < t.cols) g.ys[(size_t)(t.t0 + e) * (g.n / 128) + t.nt] = s.scale;
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                // codes as [token][64 columns]
                uint16_t *codes = reinterpret_cast<uint16_t *>(sh.stg);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i * 8 >= mine) break;
                    const int c = col0 + i * 8 + c2;
                    const float2 r = *reinterpret_cast<const float2 *>(&peak[0][c]);
                    const int slot = q * 8 + r4;
                    codes[c * 32 + (slot ^ ((c >> 1 & 3) * 8))] = (uint16_t)code2(low(acc[i][0][0]), low(acc[i][0][1]), r.x);
                    codes[(c + 1) * 32 + (slot ^ ((c >> 1 & 3) * 8))] = (uint16_t)code2(high(acc[i][0][0]), high(acc[i][0][1]), r.y);
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                for (int i = e; i < t.cols * 4; i += 256) {
                    const int c = i >> 2, part = i & 3;
                    const uint4 v = *reinterpret_cast<const uint4 *>(&codes[c * 32 + ((part * 8) ^ ((c >> 1 & 3) * 8))]);
                    if (ok) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(g.y) + (size_t)(t.t0 + c) * g.n + t.nt * 128 + rank * 64 + part * 16) = v;
                }
                // (the next tile writes codes behind several of its barriers)
            } else {
                // eight tokens at a time are turned through shared memory, so that a store covers whole pieces of consecutive columns
                const int n_col = t.nt * PR_TILE + (int)rank * 128 + q * 32;
                unsigned char *stg = sh.stg + (warp - 4) * PR_STG_WARP;
                if (ok && n_col < g.n) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int c0 = col0 + i * 8;
                        if (i * 8 >= mine || c0 >= t.cols) break;
                        if (g.out == SPICE_OUT_BF16) {
                            unsigned char *to = stg + (i & 1) * (8 * PR_PITCH);
                            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                                         ::"r"(smem_u32(to + (lane & 7) * PR_PITCH + (lane >> 3) * 16)),
                                           "r"(pack2(low(acc[i][0][0]), high(acc[i][0][0]))), "r"(pack2(low(acc[i][0][1]), high(acc[i][0][1]))),
                                           "r"(pack2(low(acc[i][1][0]), high(acc[i][1][0]))), "r"(pack2(low(acc[i][1][1]), high(acc[i][1][1]))) : "memory");
                            __syncwarp();
                            const int part = lane & 3, col = n_col + part * 8;
                            const uint4 v = *reinterpret_cast<const uint4 *>(to + r4 * PR_PITCH + part * 16);
                            if (c0 + r4 < t.cols && col < g.n)
                                *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(g.y) + (size_t)(t.t0 + c0 + r4) * g.n + col) = v;
                        } else {
                            float *to = reinterpret_cast<float *>(stg);
                            constexpr int P = PR_F32_PITCH / 4;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const uint64_t v = acc[i][r >> 1][r & 1];
                                to[c2 * P + r * 8 + r4] = low(v);
                                to[(c2 + 1) * P + r * 8 + r4] = high(v);
                            }
                            __syncwarp();
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                const int tok = p * 4 + (lane >> 3), part = lane & 7, col = n_col + part * 4;
                                float4 v = *reinterpret_cast<const float4 *>(to + tok * P + part * 4);
                                if (c0 + tok < t.cols && col < g.n) {
                                    float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(g.y) + (size_t)(t.t0 + c0 + tok) * g.n + col);
                                    if (g.out == SPICE_OUT_F32_ADD) {
                                        const float4 o = *dst;
                                        v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
                                    }
                                    *dst = v;
                                }
                            }
                            __syncwarp();
                        }
                    }
                }
                __syncwarp();   // (the buffers are free again)
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort_flag && g.status) atomicMax(g.status, (int)SPICE_ERR_TIMEOUT);
    cluster_sync();   // the pair's MMAs, copies and signals are over in both CTAs
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512));
}

// ------------------------------------------------------------------------------------------------ host side
std::atomic<uint32_t> wait_limit{WAIT_LIMIT};   // (SPICE_OPT_E4M3_WAIT_LIMIT)

// What a device is told once: the dynamic shared memory limits.
bool prepare_device(int dev) {
    static std::atomic<bool> ready[64];
    if (ready[dev].load(std::memory_order_acquire)) return true;
    auto raise = [](const void *kernel, size_t bytes) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
    };
    if (!raise((const void *)gemm_e4m3_pair_kernel<false>, PR_SMEM_BYTES) || !raise((const void *)gemm_e4m3_pair_kernel<true>, PR_SMEM_BYTES))
        return false;
    ready[dev].store(true, std::memory_order_release);
    return true;
}

template <bool SWIGLU>
spice_status launch_gemm_e4m3(GemmE4m3Args g, const uint8_t *x, const uint8_t *w, cudaStream_t st) {
    int dev = 0;
    const int sms = current_device_sms(&dev);
    if (sms <= 0 || !prepare_device(dev)) return SPICE_ERR_CUDA;
    const int w_rows = SWIGLU ? 2 * g.n : g.n;
    const int used = std::min(g.G, g.T);   // groups that can have rows
    const int rows = (g.T + used - 1) / used;
    if (rows <= 16) {
        const dim3 grid((unsigned)((g.n + 15) / 16), (unsigned)used);
        auto *kernel = rows <= 4 ? gemm_e4m3_few_kernel<1, SWIGLU> : gemm_e4m3_few_kernel<2, SWIGLU>;
        return launch_early(kernel, grid, FEW_WARPS * 32, 0, st, SWIGLU ? FEW_CLUSTER : 1, x, w, g) ? SPICE_OK : SPICE_ERR_CUDA;
    }
    g.n_tiles = SWIGLU ? g.n / 128 : (g.n + PR_TILE - 1) / PR_TILE;
    const int64_t most = ((int64_t)g.T / PR_TILE + g.G) * g.n_tiles;   // tiles there can be
    if (most > 0x3fffffff) return SPICE_ERR_UNSUPPORTED_SHAPE;
    CUtensorMap map_w, map_x[3];
    if (SWIGLU) {
        // rows of a tile in shared memory: 16 gate rows, their 16 up rows, the next 16 gate rows, ...; within 16 the even rows, then
        // the odd ones: a thread's two sums of a token are neighbours
        const uint64_t k = (uint64_t)g.k, in = (uint64_t)g.n;
        const uint64_t dims[5] = {k, 8, 2, 2 * (uint64_t)g.G, in / 16}, strides[4] = {2 * k, k, in * k, 16 * k};
        const uint32_t box[5] = {BK, 8, 2, 2, 4};
        if (!tc_encode_map5(&map_w, w, dims, strides, box, 1)) return SPICE_ERR_CUDA;
    } else if (!tc_encode_map2_bytes(&map_w, w, (uint64_t)g.G * w_rows, (uint64_t)g.k, 128)) {
        return SPICE_ERR_CUDA;
    }
    for (int i = 0; i < 3; ++i)
        if (!tc_encode_map2_bytes(&map_x[i], x, (uint64_t)g.T, (uint64_t)g.k, 64u >> i)) return SPICE_ERR_CUDA;
    const int pairs = (int)std::min<int64_t>(sms / 2, most);
    return launch_early(gemm_e4m3_pair_kernel<SWIGLU>, dim3(2 * (unsigned)pairs), PR_THREADS, PR_SMEM_BYTES, st, 2, map_w, map_x[0], map_x[1],
                        map_x[2], g) ? SPICE_OK : SPICE_ERR_CUDA;
}

bool misaligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

template <bool SWIGLU>
spice_status call_gemm_e4m3(const uint8_t *x_q, const float *x_scale, const uint8_t *w_q, const float *w_scale, const int32_t *offset,
                            int32_t n_groups, int32_t T, int32_t n, int32_t k, int32_t out, void *y, float *y_scale,
                            int32_t *device_status, void *stream) {
    if (T < 0 || n < 8 || n % 8 || k < 16 || k % 16 || n_groups < 1 || (!offset && n_groups != 1) ||
        (out != SPICE_OUT_BF16 && out != SPICE_OUT_F32 && out != SPICE_OUT_F32_ADD))
        return SPICE_ERR_INVALID_ARG;
    if (n_groups > MAX_GROUPS || k > (1 << 24) || n > (1 << 24) || T > (1 << 24) || (SWIGLU && n % 128) ||
        (int64_t)n_groups * n * (SWIGLU ? 2 : 1) > 0x7fffffffLL)
        return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    if (!x_q || !x_scale || !w_q || !w_scale || !y || (SWIGLU && !y_scale) || !aligned16(x_q) || !aligned16(w_q) || !aligned16(y) ||
        misaligned4(x_scale) || misaligned4(w_scale) || misaligned4(offset) || misaligned4(y_scale) || misaligned4(device_status))
        return SPICE_ERR_INVALID_ARG;
    GemmE4m3Args g{};
    g.xs = x_scale;
    g.ws = w_scale;
    g.offset = offset;
    g.y = y;
    g.ys = y_scale;
    g.T = T;
    g.n = n;
    g.k = k;
    g.G = n_groups;
    g.kb = (k + BK - 1) / BK;
    g.out = out;
    g.status = device_status;
    g.wait_limit = wait_limit.load(std::memory_order_relaxed);
    return launch_gemm_e4m3<SWIGLU>(g, x_q, w_q, static_cast<cudaStream_t>(stream));
}

}  // namespace

void set_gemm_e4m3_wait_limit(uint32_t polls) { wait_limit.store(polls, std::memory_order_relaxed); }

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_gemm_e4m3_blocks(const uint8_t *x_q, const float *x_scale, const uint8_t *w_q, const float *w_scale,
                                               const int32_t *offset, int32_t n_groups, int32_t T, int32_t n, int32_t k, int32_t out,
                                               void *y, int32_t *device_status, void *stream) {
    Range range_("spice_gemm_e4m3_blocks");
    return call_gemm_e4m3<false>(x_q, x_scale, w_q, w_scale, offset, n_groups, T, n, k, out, y, nullptr, device_status, stream);
}

extern "C" spice_status spice_swiglu_e4m3_blocks(const uint8_t *x_q, const float *x_scale, const uint8_t *w_gate_up_q, const float *w_scale,
                                                 const int32_t *offset, int32_t n_groups, int32_t T, int32_t inter, int32_t k,
                                                 uint8_t *act_q, float *act_scale, int32_t *device_status, void *stream) {
    Range range_("spice_swiglu_e4m3_blocks");
    return call_gemm_e4m3<true>(x_q, x_scale, w_gate_up_q, w_scale, offset, n_groups, T, inter, k, SPICE_OUT_BF16, act_q, act_scale,
                                device_status, stream);
}
