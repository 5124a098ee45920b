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
// tiles of 256 tokens x 256 weight rows, persistent.
#include <cuda_fp8.h>

#include <algorithm>

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
    int32_t sectors;         // rows of y begin on 32-byte boundaries
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
__device__ __forceinline__ void add_scaled2(uint64_t &sum, uint32_t lo, uint32_t hi, uint64_t scale) {
    asm("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(sum) : "r"(lo), "r"(hi), "l"(scale));
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

// 32 bytes; whole: they begin on a boundary of 32 bytes
__device__ __forceinline__ void store_sector(void *to, const uint32_t (&v)[8], int32_t whole) {
    if (whole) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        reinterpret_cast<uint4 *>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4 *>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
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
constexpr int PR_THREADS = 384, PR_EPI_WARPS = 8;
constexpr uint32_t PR_STAGES = 6;
constexpr int PR_TILE = 256;                      // tokens of a pair's tile (128 per CTA), and its accumulator columns
constexpr int PR_HALF_BYTES = 128 * BK;           // a CTA's half of one operand
constexpr int PR_STAGE_BYTES = 2 * PR_HALF_BYTES;
constexpr int PR_GROUP_M = 16;                    // token tiles that share a sweep over the weight tiles
// The sums of a tile take 128 registers of each epilogue thread: the four warps that copy and multiply give theirs up.
constexpr int PR_REGS_HELPERS = 72, PR_REGS_EPILOGUE = 216;
static_assert(PR_REGS_HELPERS + 2 * PR_REGS_EPILOGUE <= 3 * (65536 / PR_THREADS / 8 * 8), "what the block is launched with");

struct PairShared {
    float peak[2][128];                           // SwiGLU: largest magnitude of a token's columns, per half of them
    int32_t first[MAX_GROUPS + 1];                // tiles before each group
    alignas(8) unsigned long long full[PR_STAGES], empty[PR_STAGES], tmem_full[2], tmem_empty[2], mma_drain[2];
    uint32_t tmem_base;
    int abort_flag;
};
constexpr size_t PR_SMEM_BYTES = sizeof(PairShared) + (size_t)PR_STAGES * PR_STAGE_BYTES + 1024;
static_assert(PR_SMEM_BYTES <= 232448, "what a block can have");

struct Tile {
    int group, t0, rows, nt;   // first token, tokens, weight tile
};

// Tiles are numbered group by group; within a group sweeps of up to PR_GROUP_M token tiles, the token tile fastest, so that
// pairs working at the same time share both operands in L2.  The group only moves forward.
__device__ __forceinline__ Tile find_tile(const PairShared &sh, const GemmE4m3Args &g, int tile, int &group) {
    while (tile >= sh.first[group + 1]) ++group;
    const int begin = g.offset ? load_s32(g.offset + group) : 0, m = (g.offset ? load_s32(g.offset + group + 1) : g.T) - begin;
    const int in = tile - sh.first[group];
    const int per_sweep = PR_GROUP_M * g.n_tiles, sweep = in / per_sweep, r = in - sweep * per_sweep;
    const int mt0 = sweep * PR_GROUP_M, left = min(PR_GROUP_M, (m + PR_TILE - 1) / PR_TILE - mt0);
    const int mt = mt0 + r % left;
    return Tile{group, begin + mt * PR_TILE, min(PR_TILE, m - mt * PR_TILE), r / left};
}
// Rows of a CTA's half of the tile as they are copied.  Some always are: a copying thread that the products do not wait for
// could fall two uses of a stage behind, and the parity of a barrier would no longer tell it which use is meant.
__device__ __forceinline__ int copied(int rows, int rank) { return (min(max(rows - rank * 128, 1), 128) + 15) & ~15; }

template <bool SWIGLU>
__global__ void __launch_bounds__(PR_THREADS, 1)
    gemm_e4m3_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x128,
                          const __grid_constant__ CUtensorMap map_x16, const GemmE4m3Args g) {
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    PairShared &sh = *reinterpret_cast<PairShared *>(ring + PR_STAGES * PR_STAGE_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    volatile int *abort_flag = &sh.abort_flag;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < PR_STAGES; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);    // used in the even CTA: both CTAs' copies report there
            mbar_init(smem_u32(&sh.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh.tmem_full[b]), 1);
            mbar_init(smem_u32(&sh.tmem_empty[b]), 2 * PR_EPI_WARPS);   // used in the even CTA: the epilogue warps of both
            mbar_init(smem_u32(&sh.mma_drain[b]), 1);
        }
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

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_HELPERS));
        if ((warp == 0 || warp == 3) && lane == 0) {
            // one of the two brings the weights, the other the tokens: what a thread does for a block takes it some hundred cycles
            const uint32_t empty0 = smem_u32(&sh.empty[0]), full0 = smem_u32(&sh.full[0]);
            uint32_t s = 0, phase = 1, filled = 0, limit = g.wait_limit;
            int group = 0;
            for (int tile = pair; tile < n_tiles && limit != 0; tile += pairs) {
                const Tile t = find_tile(sh, g, tile, group);
                // (SwiGLU: the even CTA brings the gate rows, the odd one the up rows)
                const int row = warp != 0 ? t.t0 + rank * 128 : SWIGLU ? (2 * t.group + rank) * g.n + t.nt * 128 : t.group * g.n + t.nt * PR_TILE + rank * 128;
                const int x_rows = copied(t.rows, rank);
                const uint32_t bytes = 2 * PR_HALF_BYTES + (x_rows + copied(t.rows, rank ^ 1)) * BK;
                for (int k0 = 0; k0 < g.k; k0 += BK) {
                    mbar_wait_quick(empty0 + s * 8, phase, abort_flag, limit);
                    if (limit == 0) break;
                    const uint32_t full = map_to_cta(full0 + s * 8, 0), dst = smem_u32(ring) + s * PR_STAGE_BYTES;
                    if (warp == 0) {
                        if (rank == 0) mbar_expect_tx(full0 + s * 8, bytes);
                        tma_load_2d_pair(dst + PR_HALF_BYTES, &map_w, k0, row, full);
                    } else if (x_rows == 128) {
                        tma_load_2d_pair(dst, &map_x128, k0, row, full);
                    } else {
                        for (int done = 0; done < x_rows; done += 16) tma_load_2d_pair(dst + done * BK, &map_x16, k0, row + done, full);
                    }
                    filled = min(filled + 1, PR_STAGES);
                    if (++s == PR_STAGES) {
                        s = 0;
                        phase ^= 1;
                    }
                }
            }
            // a CTA ends when the stages it filled have been read by the MMAs: nothing of it is in flight then, neither a
            // copy nor a release of a stage (also after an abort, within the limit: copies have long landed by then)
            for (uint32_t left = filled; left > 0; --left) {
                const uint32_t back = s >= left ? 0u : 1u;   // the stage filled `left` blocks ago: in this round of the ring, or the one before
                if (!mbar_drain(empty0 + (s + back * PR_STAGES - left) * 8, phase ^ 1 ^ back)) {
                    *abort_flag = 1;
                    break;
                }
            }
        } else if ((warp == 1 || warp == 2) && rank == 0 && lane == 0) {
            // Every other block of the reduction is issued by the other of these warps, into its own accumulator: issuing a block
            // takes longer than its products do.
            static_assert(PR_STAGES % 2 == 0, "a stage always belongs to the same warp");
            constexpr uint32_t idesc = make_idesc_e4m3(256, PR_TILE);
            const uint32_t buf = warp - 1, d_tmem = tmem_base + buf * PR_TILE;
            const uint32_t tmem_empty = smem_u32(&sh.tmem_empty[buf]), tmem_full = smem_u32(&sh.tmem_full[buf]);
            const uint32_t full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
            const uint64_t desc0 = make_desc(smem_u32(ring));
            uint32_t s = buf, phase = 0, tmem_phase = 1, limit = g.wait_limit;
            // blocks of all this pair's tiles that are this warp's
            const uint32_t total = (uint32_t)(n_tiles > pair ? (n_tiles - pair + pairs - 1) / pairs : 0) * (uint32_t)g.kb;
            for (uint32_t left = (total + 1 - buf) / 2; left > 0; --left) {
                mbar_wait_quick(tmem_empty, tmem_phase, abort_flag, limit);
                mbar_wait_quick(full0 + s * 8, phase, abort_flag, limit);
                if (limit == 0) break;
                tc_fence_after();
                const uint64_t da = desc0 + s * (PR_STAGE_BYTES >> 4), db = da + (PR_HALF_BYTES >> 4);
#pragma unroll
                for (int k = 0; k < BK / 32; ++k) tc_mma_f8_pair(d_tmem, da + 2 * k, db + 2 * k, idesc, k ? 1u : 0u);
                tc_commit_pair(empty0 + s * 8, 3u);
                tc_commit_pair(tmem_full, 3u);
                tmem_phase ^= 1;
                s += 2;
                if (s >= PR_STAGES) {
                    s -= PR_STAGES;
                    phase ^= 1;
                }
            }
            tc_commit_pair_local(smem_u32(&sh.mma_drain[buf]));
            if (!mbar_drain(smem_u32(&sh.mma_drain[buf]), 0)) *abort_flag = 1;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PR_REGS_EPILOGUE));
        // ---------------- epilogue: warp w reads TMEM lanes 32*(w%4) .. +31 = tokens of this CTA's half of the tile, a token per
        // thread; the two warps of a quarter take 128 columns each (SwiGLU: 64 gate columns and their up columns), which are one
        // block of weight rows: a thread's sums of a block all have the same scale.
        const int q = warp & 3, h = warp >= 8 ? 1 : 0;
        const int row_blocks = ((SWIGLU ? 2 * g.n : g.n) + 127) / 128;
        const uint32_t full0 = smem_u32(&sh.tmem_full[0]), empty0 = map_to_cta(smem_u32(&sh.tmem_empty[0]), 0);
        const uint32_t tm0 = tmem_base + ((uint32_t)(q * 32) << 16) + h * (SWIGLU ? 64 : 128);
        uint32_t it = 0;
        uint32_t limit = g.wait_limit;   // 0 after an expired wait: a warp only keeps the others' barriers
        int group = 0;
        for (int tile = pair; tile < n_tiles; tile += pairs) {
            const Tile t = find_tile(sh, g, tile, group);
            const int rows = t.rows - rank * 128 - q * 32;              // of this warp
            const int row = t.t0 + rank * 128 + q * 32 + lane;          // of this thread
            const int nb = SWIGLU ? t.nt : min(t.nt * 2 + h, row_blocks - 1);
            const float *ws = g.ws + ((size_t)t.group * row_blocks + nb) * g.kb, *wu = ws + (size_t)(g.n / 128) * g.kb;
            const float *xs = g.xs + (size_t)(lane < rows ? row : t.t0) * g.kb;
            uint64_t acc[64];   // two columns each
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0;
            float x = load_f32(xs), w = load_f32(ws), u = SWIGLU ? load_f32(wu) : 0.0f;   // a block ahead
#pragma unroll 1
            for (int kb = 0; kb < g.kb; ++kb, ++it) {
                const uint32_t buf = it & 1, tm = tm0 + buf * PR_TILE;
                const float sw = x * w, su = SWIGLU ? x * u : sw;
                const int ahead = min(kb + 1, g.kb - 1);
                x = load_f32(xs + ahead);
                w = load_f32(ws + ahead);
                if (SWIGLU) u = load_f32(wu + ahead);
                mbar_wait_quick(full0 + buf * 8, (it >> 1) & 1, abort_flag, limit);
                tc_fence_after();
                if (rows > 0) {
#pragma unroll
                    for (int ch = 0; ch < 8; ++ch) {
                        uint32_t v[16];
                        const int off = (SWIGLU && ch >= 4 ? 64 : 0) + ch * 16;
                        tc_ld16(tm + off, v);
                        tc_wait_ld();
                        asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]));
                        if (ch == 7) {   // the last columns are in registers: the buffer is free
                            tc_fence_before();
                            mbar_arrive_cluster_tmem(empty0 + buf * 8, lane);
                        }
                        const float f = SWIGLU && ch >= 4 ? su : sw;
#pragma unroll
                        for (int i = 0; i < 8; ++i) add_scaled2(acc[ch * 8 + i], v[2 * i], v[2 * i + 1], pair2(f, f));
                    }
                } else {
                    mbar_arrive_cluster_tmem(empty0 + buf * 8, lane);
                }
            }
            // a thread writes its token's columns, whole sectors at a time
            const bool in = limit != 0 && lane < rows;
            if constexpr (SWIGLU) {
                // activations into the gate columns' sums; a block is the columns of both warps of the quarter
                float big = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float a = silu_times(low(acc[i]), low(acc[32 + i])), b = silu_times(high(acc[i]), high(acc[32 + i]));
                    acc[i] = pair2(a, b);
                    big = max_magnitude(max_magnitude(big, a), b);
                }
                sh.peak[h][q * 32 + lane] = big;
                asm volatile("bar.sync %0, 64;" ::"r"(1 + q) : "memory");
                const OutScale s(max_magnitude(big, sh.peak[h ^ 1][q * 32 + lane]));
                asm volatile("bar.sync %0, 64;" ::"r"(1 + q) : "memory");   // (both have read before either writes again)
                if (in) {
                    if (h == 0) g.ys[(size_t)row * (g.n / 128) + t.nt] = s.scale;
                    uint8_t *to = static_cast<uint8_t *>(g.y) + (size_t)row * g.n + t.nt * 128 + h * 64;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t c[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint64_t a = acc[k * 16 + 2 * i], b = acc[k * 16 + 2 * i + 1];
                            c[i] = code2(low(a), high(a), s.r) | code2(low(b), high(b), s.r) << 16;
                        }
                        store_sector(to + k * 32, c, g.sectors);
                    }
                }
            } else if (in) {
                const int col0 = t.nt * PR_TILE + h * 128;
                if (g.out == SPICE_OUT_BF16) {
                    __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(g.y) + (size_t)row * g.n + col0;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        if (col0 + c * 16 >= g.n) break;
                        uint32_t v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = pack2(low(acc[c * 8 + i]), high(acc[c * 8 + i]));
                        if (col0 + c * 16 + 16 <= g.n) store_sector(to + c * 16, v, g.sectors);
                        else *reinterpret_cast<uint4 *>(to + c * 16) = make_uint4(v[0], v[1], v[2], v[3]);   // (n is a multiple of 8)
                    }
                } else {
                    float *to = static_cast<float *>(g.y) + (size_t)row * g.n + col0;
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        if (col0 + c * 8 >= g.n) break;
                        float f[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f[2 * i] = low(acc[c * 4 + i]);
                            f[2 * i + 1] = high(acc[c * 4 + i]);
                        }
                        if (g.out == SPICE_OUT_F32_ADD) {
                            const float4 a = *reinterpret_cast<const float4 *>(to + c * 8), b = *reinterpret_cast<const float4 *>(to + c * 8 + 4);
                            const float o[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                            for (int i = 0; i < 8; ++i) f[i] += o[i];
                        }
                        uint32_t v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(f[i]);
                        store_sector(to + c * 8, v, g.sectors);
                    }
                }
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
    const int row_bytes = SWIGLU ? 1 : g.out == SPICE_OUT_BF16 ? 2 : 4;
    g.sectors = ((reinterpret_cast<uintptr_t>(g.y) | (uintptr_t)g.n * row_bytes) & 31u) == 0;
    const int64_t most = ((int64_t)g.T / PR_TILE + g.G) * g.n_tiles;   // tiles there can be
    if (most > 0x3fffffff) return SPICE_ERR_UNSUPPORTED_SHAPE;
    CUtensorMap map_w, map_x128, map_x16;
    if (!tc_encode_map2_bytes(&map_w, w, (uint64_t)g.G * w_rows, (uint64_t)g.k, 128) ||
        !tc_encode_map2_bytes(&map_x128, x, (uint64_t)g.T, (uint64_t)g.k, 128) ||
        !tc_encode_map2_bytes(&map_x16, x, (uint64_t)g.T, (uint64_t)g.k, 16))
        return SPICE_ERR_CUDA;
    const int pairs = (int)std::min<int64_t>(sms / 2, most);
    return launch_early(gemm_e4m3_pair_kernel<SWIGLU>, dim3(2 * (unsigned)pairs), PR_THREADS, PR_SMEM_BYTES, st, 2, map_w, map_x128, map_x16,
                        g) ? SPICE_OK : SPICE_ERR_CUDA;
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
