// Products of 8-bit integer rows with a scale per token and per output channel, on the 5th-generation tensor cores:
//
//   y[t, n] = ( sum_k x[t,k] w[n,k] ) * x_scale[t] * w_scale[n]                        (bf16, fp32, or added to fp32)
//   SwiGLU:   g, u = the products with the gate and the up rows;   act[t, i] = bf16( g / (1 + e^-g) * u )
//
// The sum is an integer and exact (k <= 131056: 2^14 k < 2^31), so neither the order of the additions nor a split of the
// reduction changes a bit; one rounding when it becomes fp32, one per scale, one to bf16.
//
// Three kernels.  A handful of tokens: straight from global memory into registers, the shortest chain of latencies.  Few
// tokens: every weight byte is used for few products and the call is bound by streaming the weights, so
// the weight rows are the M operand, the tokens the N operand (as in the fused decode kernel), and the reduction is split
// over the CTAs of a cluster so that narrow layers still fill the GPU; the cluster adds its partial sums through
// distributed shared memory, no workspace and no atomics.  Many tokens: pairs of CTAs work on 256 x 256 tiles
// (cta_group::2: each CTA loads half of either operand), persistent, accumulators double-buffered in TMEM.
#include <algorithm>
#include <mutex>

#include "entry.cuh"
#include "spice_internal.cuh"
#include "tc_device.cuh"

namespace spice {

namespace {

using namespace tcdev;

constexpr int BK = 128;                 // bytes = elements of the reduction per pipeline stage: one swizzle span
constexpr int MAX_K = 131056;

struct GemmI8Args {
    const float *xs, *ws;   // [T], [n] (SwiGLU: [2 inter])
    void *y;                // [T, n] (SwiGLU: [T, inter])
    int32_t T, n, k;        // n: columns of y
    int32_t out;            // SPICE_OUT_*
    int32_t *status;        // optional
    uint32_t wait_limit;    // polls after which a wait inside a kernel gives up
    // few tokens
    int32_t split, stages, cols;   // CTAs (pairs) along the reduction; ring stages, token columns of a tile (multiple of 16)
    // many tokens
    int32_t m_tiles, n_tiles;
};

// (fast exponential and quotient: a few 2^-23 for |g| of some units, the result is rounded to bf16 right after)
__device__ __forceinline__ float silu_times(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
}

// four consecutive outputs of one token
__device__ __forceinline__ void store4(const GemmI8Args &g, size_t at, float4 v) {
    if (g.out == SPICE_OUT_BF16) {
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(g.y) + at) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
        return;
    }
    float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(g.y) + at);
    if (g.out == SPICE_OUT_F32_ADD) {
        const float4 o = *dst;
        v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
    }
    *dst = v;
}

// ------------------------------------------------------------------------------------------------ a handful of tokens
// A block multiplies 16 weight rows (SwiGLU: 8 gate rows and their up rows) with all tokens; its warps share the reduction
// in pieces of 64.  The weights go from global memory straight into the registers of warp-wide 16 x 8 x 32 products: a lane
// reads 16 consecutive bytes of its row, and since both operands are read alike, the order of the reduction inside a piece
// does not matter.  The call is over before the tensor-memory kernel has its first tile (descriptors, barriers, TMEM and the
// cluster's sums are a chain of some 6 us).  What limits it is the reads of the tokens, which every block repeats.
constexpr int FEW_MAX_TOKENS = 32;

// 16 bytes that are read once (weights), or again by other warps of the SM (tokens)
__device__ __forceinline__ int4 load_once(const int4 *p) {
    int4 v;
    asm volatile("ld.global.cs.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int4 load_shared_by_warps(const int4 *p) {
    int4 v;
    asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int NT, int NW, int UN, bool DEAL, bool SWIGLU>
__global__ void __launch_bounds__(NW * 32) gemm_i8_few_kernel(const int8_t *x, const int8_t *w,
                                                              const GemmI8Args g) {
    __shared__ int32_t red[NW][NT * 8][16 + 4];   // (padded: the 8 rows of a warp's store fall into different banks)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gq = lane >> 2, c = lane & 3;
    const int n0 = blockIdx.x * (SWIGLU ? 8 : 16);
    const int r0 = n0 + gq, r1 = SWIGLU ? g.n + n0 + gq : n0 + gq + 8;
    const bool in1 = SWIGLU || n0 + 8 < g.n;                             // (n is a multiple of 8)
    const int4 *w0 = reinterpret_cast<const int4 *>(w + (size_t)r0 * g.k);
    const int4 *w1 = reinterpret_cast<const int4 *>(w + (size_t)(in1 ? r1 : r0) * g.k);
    const int4 *x4 = reinterpret_cast<const int4 *>(x);
    const int nv = g.k >> 4, pieces = (nv + 3) >> 2;
    // DEAL: pieces are dealt out one at a time, so that every warp has the same share of a short reduction; of a long one a
    // warp takes UN pieces side by side, whole lines of DRAM (dealt out / side by side, us: 8 tokens 2048 x 2816 3.0 / 4.0, 4096
    // x 11008 12.1 / 11.7, one token 4096 x 11008 11.9 / 11.2; 16 tokens 4096 x 11008 12.2 / 13.3: there it loses).
    int32_t acc[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0;
    grid_dependency();
    const int4 zero = make_int4(0, 0, 0, 0);
    for (int p0 = DEAL ? warp : warp * UN; p0 < pieces; p0 += NW * UN) {
        int4 a0[UN], a1[UN], b[UN][NT];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int v = (p0 + u * (DEAL ? NW : 1)) * 4 + c;
            a0[u] = v < nv ? load_once(w0 + v) : zero;
            a1[u] = v < nv ? load_once(w1 + v) : zero;
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int v = (p0 + u * (DEAL ? NW : 1)) * 4 + c;
#pragma unroll
            for (int i = 0; i < NT; ++i) b[u][i] = v < nv && i * 8 + gq < g.T ? load_shared_by_warps(x4 + (size_t)(i * 8 + gq) * nv + v) : zero;
        }
#pragma unroll
        for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                             : "+r"(acc[i][0]), "+r"(acc[i][1]), "+r"(acc[i][2]), "+r"(acc[i][3])
                             : "r"(a0[u].x), "r"(a1[u].x), "r"(a0[u].y), "r"(a1[u].y), "r"(b[u][i].x), "r"(b[u][i].y));
                asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                             : "+r"(acc[i][0]), "+r"(acc[i][1]), "+r"(acc[i][2]), "+r"(acc[i][3])
                             : "r"(a0[u].z), "r"(a1[u].z), "r"(a0[u].w), "r"(a1[u].w), "r"(b[u][i].z), "r"(b[u][i].w));
            }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {   // rows gq, gq + 8 x tokens 2c, 2c + 1
        red[warp][i * 8 + 2 * c][gq] = acc[i][0];
        red[warp][i * 8 + 2 * c + 1][gq] = acc[i][1];
        red[warp][i * 8 + 2 * c][gq + 8] = acc[i][2];
        red[warp][i * 8 + 2 * c + 1][gq + 8] = acc[i][3];
    }
    __syncthreads();
    constexpr int ROWS = SWIGLU ? 8 : 16;
    for (int i = threadIdx.x; i < g.T * ROWS; i += NW * 32) {
        const int t = i / ROWS, r = i % ROWS;
        if (n0 + r >= g.n) continue;
        int32_t s = 0, u = 0;
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            s += red[q][t][r];
            if (SWIGLU) u += red[q][t][r + 8];
        }
        const float xs = g.xs[t];
        float v = (float)s * xs * g.ws[n0 + r];
        if (SWIGLU) v = silu_times(v, (float)u * xs * g.ws[g.n + n0 + r]);
        const size_t at = (size_t)t * g.n + n0 + r;
        if (g.out == SPICE_OUT_BF16) static_cast<__nv_bfloat16 *>(g.y)[at] = __float2bfloat16_rn(v);
        else if (g.out == SPICE_OUT_F32) static_cast<float *>(g.y)[at] = v;
        else static_cast<float *>(g.y)[at] += v;
    }
}

// ------------------------------------------------------------------------------------------------ few tokens
constexpr int SK_THREADS = 256, SK_MAX_STAGES = 12, SK_MAX_SPLIT = 8;
constexpr int SK_W_BYTES = 128 * BK;
constexpr int SK_MAX_SMEM = 225 * 1024;

struct SkinnyShared {
    alignas(8) unsigned long long full[SK_MAX_STAGES], empty[SK_MAX_STAGES], done;
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float ws[128];   // of the tile's weight rows
    float xs[128];               // of its tokens
};

__device__ __forceinline__ int4 ld_cluster4(uint32_t cluster_addr) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(cluster_addr));
    return v;
}

// grid: x = row tiles * split (a cluster = one row tile), y = token tiles.  Row tile: 128 weight rows (SwiGLU: 64 gate
// rows and their 64 up rows).
template <bool SWIGLU>
__global__ void __launch_bounds__(SK_THREADS) gemm_i8_skinny_kernel(const __grid_constant__ CUtensorMap map_w,
                                                                    const __grid_constant__ CUtensorMap map_x, const GemmI8Args g) {
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ SkinnyShared sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh.abort_flag;
    const int split = g.split, rank = blockIdx.x % split, tile = blockIdx.x / split;
    const int cols = g.cols, stages = g.stages, stage_bytes = SK_W_BYTES + cols * BK;
    const int n0 = tile * (SWIGLU ? 64 : 128), t0 = blockIdx.y * cols;
    const int kblocks = (g.k + BK - 1) / BK;
    const int kb0 = kblocks * rank / split, n_it = kblocks * (rank + 1) / split - kb0;
    uint32_t tmem_cols = 32;
    while (tmem_cols < (uint32_t)cols) tmem_cols *= 2;

    auto load_stage = [&](int it) {
        const int s = it % stages, k0 = (kb0 + it) * BK;
        const uint32_t full = smem_u32(&sh.full[s]), dst = smem_u32(ring + s * stage_bytes);
        mbar_expect_tx(full, stage_bytes);
        tma_load_2d(dst, &map_w, k0, n0, full);
        if (SWIGLU) tma_load_2d(dst + SK_W_BYTES / 2, &map_w, k0, g.n + n0, full);
        tma_load_2d(dst + SK_W_BYTES, &map_x, k0, t0, full);
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);
            mbar_init(smem_u32(&sh.empty[s]), 1);
        }
        mbar_init(smem_u32(&sh.done), 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
        grid_dependency();
        // the first copies leave before the block is set up: a short call is a chain of latencies
        for (int it = 0; it < min(stages, n_it); ++it) load_stage(it);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(tmem_cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    grid_dependency();

    if (warp == 0 && lane == 0) {
        int it = min(stages, n_it);
        for (; it < n_it; ++it) {
            if (!mbar_wait(smem_u32(&sh.empty[it % stages]), ((it / stages) & 1) ^ 1, abort_flag, g.wait_limit)) break;
            load_stage(it);
        }
        // every stage that was armed has landed before the ring is reused or the CTA ends
        for (int j = it > stages ? it - stages : 0; j < it; ++j)
            if (!mbar_drain(smem_u32(&sh.full[j % stages]), (j / stages) & 1)) *abort_flag = 1;
    } else if (warp == 1 && lane == 0) {
        const uint32_t idesc = make_idesc_i8(128, cols);
        for (int it = 0; it < n_it; ++it) {
            const int s = it % stages;
            if (!mbar_wait(smem_u32(&sh.full[s]), (it / stages) & 1, abort_flag, g.wait_limit)) break;
            tc_fence_after();
            const uint32_t w0 = smem_u32(ring + s * stage_bytes);
            const uint64_t dw = make_desc(w0), dx = make_desc(w0 + SK_W_BYTES);
#pragma unroll
            for (int k = 0; k < BK / 32; ++k) tc_mma_i8(tmem, dw + 2 * k, dx + 2 * k, idesc, (it | k) ? 1u : 0u);
            tc_commit(smem_u32(&sh.empty[s]));
        }
        tc_commit(smem_u32(&sh.done));
        // (one thread polls, the others wait in hardware: pollers slow the two that work)
        if (!mbar_drain(smem_u32(&sh.done), 0)) *abort_flag = 1;
    }
    __syncwarp();
    if (threadIdx.x >= 128) {   // the scales arrive while the products run
        const int r = threadIdx.x - 128, row = SWIGLU ? n0 + (r & 63) : n0 + r;
        sh.ws[r] = row < g.n ? g.ws[row + (SWIGLU && r >= 64 ? g.n : 0)] : 0.0f;
        for (int c = r; c < cols; c += 128) sh.xs[c] = t0 + c < g.T ? g.xs[t0 + c] : 0.0f;
    }
    __syncthreads();   // the products are done, and the producer has seen its last copies land: the ring is free
    tc_fence_after();

    // ---- sums into shared memory, [token column][128 rows]
    const int ncol = min(cols, g.T - t0);
    int32_t *red = reinterpret_cast<int32_t *>(ring);
    const int q = warp & 3;   // a warp reads the TMEM lanes of its quarter; the two warps of a quarter share the columns
    for (int c = (warp >> 2) * 16; c < ncol; c += 32) {
        uint32_t v[16];
        tc_ld16(tmem + ((uint32_t)(q * 32) << 16) + c, v);
        tc_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < ncol) red[(c + j) * 128 + q * 32 + lane] = (int32_t)v[j];
    }
    tc_fence_before();
    if (split > 1) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));

    // ---- every CTA of the cluster finishes its share of the tile, four rows of a column at a time
    constexpr int QUADS = SWIGLU ? 16 : 32;
    const int items = ncol * QUADS;
    const uint32_t red_s = smem_u32(red);
    const int4 *red4 = reinterpret_cast<const int4 *>(red);
    auto at_own = [](int c, int row) { return c * 32 + row / 4; };
    for (int i = items * rank / split + threadIdx.x; i < items * (rank + 1) / split; i += SK_THREADS) {
        const int c = i / QUADS, row = (i % QUADS) * 4;
        if (n0 + row >= g.n) continue;
        int4 a = make_int4(0, 0, 0, 0), b = make_int4(0, 0, 0, 0);
        const uint32_t at = red_s + (uint32_t)(c * 128 + row) * 4;
        if (split == 1) {
            a = red4[at_own(c, row)];
            if (SWIGLU) b = red4[at_own(c, row + 64)];
        } else {
            // all loads leave before the first is used: a peer's shared memory is some hundred cycles away
            int4 p[SK_MAX_SPLIT], u[SWIGLU ? SK_MAX_SPLIT : 1];
#pragma unroll
            for (int r = 0; r < SK_MAX_SPLIT; ++r) {
                p[r] = r < split ? ld_cluster4(map_to_cta(at, (uint32_t)r)) : make_int4(0, 0, 0, 0);
                if (SWIGLU) u[r] = r < split ? ld_cluster4(map_to_cta(at + 64 * 4, (uint32_t)r)) : make_int4(0, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < SK_MAX_SPLIT; ++r) {
                a = make_int4(a.x + p[r].x, a.y + p[r].y, a.z + p[r].z, a.w + p[r].w);
                if (SWIGLU) b = make_int4(b.x + u[r].x, b.y + u[r].y, b.z + u[r].z, b.w + u[r].w);
            }
        }
        const float xs = sh.xs[c];
        const float4 w4 = *reinterpret_cast<const float4 *>(&sh.ws[row]);
        float4 v = make_float4((float)a.x * xs * w4.x, (float)a.y * xs * w4.y, (float)a.z * xs * w4.z, (float)a.w * xs * w4.w);
        if (SWIGLU) {
            const float4 u4 = *reinterpret_cast<const float4 *>(&sh.ws[64 + row]);
            v = make_float4(silu_times(v.x, (float)b.x * xs * u4.x), silu_times(v.y, (float)b.y * xs * u4.y),
                            silu_times(v.z, (float)b.z * xs * u4.z), silu_times(v.w, (float)b.w * xs * u4.w));
        }
        store4(g, (size_t)(t0 + c) * g.n + n0 + row, v);
    }
    if (threadIdx.x == 0 && sh.abort_flag && g.status) atomicMax(g.status, (int)SPICE_ERR_TIMEOUT);
    if (split > 1) cluster_sync();   // nobody leaves while a peer reads its sums
}

// ------------------------------------------------------------------------------------------------ many tokens
constexpr int PR_THREADS = 320, PR_STAGES = 6, PR_EPI_WARPS = 8;
constexpr int PR_TILE = 256;                                   // tokens and accumulator columns of a pair's tile
constexpr int PR_HALF_BYTES = 128 * BK;                        // a CTA's half of one operand
constexpr int PR_STAGE_BYTES = 2 * PR_HALF_BYTES;
constexpr int PR_PITCH = 80;                                   // 64 B of a row's outputs + 16: 16-byte accesses do not collide
constexpr int PR_STG_WARP = 32 * PR_PITCH;                     // an epilogue warp's transposition buffer
static_assert(PR_TILE * 128 * 4 <= PR_STAGES * PR_STAGE_BYTES, "the sums fit in the ring");
constexpr size_t PR_SMEM = (size_t)PR_STAGES * PR_STAGE_BYTES + PR_EPI_WARPS * PR_STG_WARP + 1024;
constexpr int PR_GROUP_M = 16;                                 // token tiles that share a sweep over the weight tiles

struct PairShared {
    alignas(8) unsigned long long full[PR_STAGES], empty[PR_STAGES], tmem_full[2], tmem_empty[2], mma_drain;
    uint32_t tmem_base;
    int abort_flag, gave_up;
    alignas(16) float ws[2][PR_TILE];   // channel scales of the tile (SwiGLU: gate, then up), per accumulator buffer
};

// tile number -> token tile, weight tile: groups of PR_GROUP_M token tiles, within a group the token tile runs fastest, so
// that pairs working at the same time share both operands in L2
__device__ __forceinline__ void pair_tile(const GemmI8Args &g, int tile, int &mt, int &nt) {
    const int per_group = PR_GROUP_M * g.n_tiles;
    const int grp = tile / per_group, first = grp * PR_GROUP_M;
    const int width = min(PR_GROUP_M, g.m_tiles - first);
    const int in = tile - grp * per_group;
    mt = first + in % width;
    nt = in / width;
}

// A warp's part of a tile: 32 tokens (row0 ..), 64 bytes of outputs at a time, every other piece of the columns [first, last).
// load(c, v): the integer sums of columns c .. of this lane's token.  A lane holds one token's outputs; they are turned
// through shared memory so that a store covers whole 16-byte pieces of consecutive columns.
template <bool SWIGLU, typename Load>
__device__ __forceinline__ void pair_store(const GemmI8Args &g, int row0, float xs, int col0, int first, int last, const float *ws,
                                           unsigned char *stg, int lane, Load load) {
    const float4 *w4 = reinterpret_cast<const float4 *>(ws), *u4 = w4 + 32;
    if (SWIGLU || g.out == SPICE_OUT_BF16) {
#pragma unroll 1
        for (int c = first; c < last; c += 64) {
            if (col0 + c >= g.n) break;
            uint32_t v[32], u[SWIGLU ? 32 : 1];
            load(c, v);
            if constexpr (SWIGLU) load(128 + c, u);
            tc_wait_ld();
            uint32_t pk[16];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 w = w4[c / 4 + j];
                float a[4] = {(float)(int32_t)v[4 * j] * xs * w.x, (float)(int32_t)v[4 * j + 1] * xs * w.y,
                              (float)(int32_t)v[4 * j + 2] * xs * w.z, (float)(int32_t)v[4 * j + 3] * xs * w.w};
                if constexpr (SWIGLU) {
                    const float4 z = u4[c / 4 + j];
                    a[0] = silu_times(a[0], (float)(int32_t)u[4 * j] * xs * z.x);
                    a[1] = silu_times(a[1], (float)(int32_t)u[4 * j + 1] * xs * z.y);
                    a[2] = silu_times(a[2], (float)(int32_t)u[4 * j + 2] * xs * z.z);
                    a[3] = silu_times(a[3], (float)(int32_t)u[4 * j + 3] * xs * z.w);
                }
                pk[2 * j] = pack2(a[0], a[1]);
                pk[2 * j + 1] = pack2(a[2], a[3]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<uint4 *>(stg + lane * PR_PITCH + k * 16) = make_uint4(pk[4 * k], pk[4 * k + 1], pk[4 * k + 2], pk[4 * k + 3]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = i * 8 + (lane >> 2), part = lane & 3, col = col0 + c + part * 8;
                const uint4 val = *reinterpret_cast<const uint4 *>(stg + rr * PR_PITCH + part * 16);
                if (row0 + rr < g.T && col < g.n)
                    *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(g.y) + (size_t)(row0 + rr) * g.n + col) = val;
            }
            __syncwarp();
        }
    } else {
#pragma unroll 1
        for (int c = first; c < last; c += (c & 16) ? 48 : 16) {   // (the same 32 columns as above, 16 at a time)
            if (col0 + c >= g.n) break;
            uint32_t v[16];
            load(c, v);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 w = w4[c / 4 + j];
                *reinterpret_cast<float4 *>(stg + lane * PR_PITCH + j * 16) =
                    make_float4((float)(int32_t)v[4 * j] * xs * w.x, (float)(int32_t)v[4 * j + 1] * xs * w.y,
                                (float)(int32_t)v[4 * j + 2] * xs * w.z, (float)(int32_t)v[4 * j + 3] * xs * w.w);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rr = i * 8 + (lane >> 2), part = lane & 3, col = col0 + c + part * 4;
                const float4 val = *reinterpret_cast<const float4 *>(stg + rr * PR_PITCH + part * 16);
                if (row0 + rr < g.T && col < g.n) store4(g, (size_t)(row0 + rr) * g.n + col, val);
            }
            __syncwarp();
        }
    }
}

// SPLIT: the reduction of a tile is shared by the g.split pairs of a cluster (one tile per cluster): each pair leaves its sums in
// its shared memory and finishes its share of the columns with those of the others.
template <bool SWIGLU, bool SPLIT>
__global__ void __launch_bounds__(PR_THREADS, 1)
    gemm_i8_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const GemmI8Args g) {
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char *stage_base = ring + PR_STAGES * PR_STAGE_BYTES;
    __shared__ PairShared sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank() & 1u, part = SPLIT ? cluster_rank() >> 1 : 0u, leader = 2 * part;
    const uint32_t pair_mask = 3u << leader;
    volatile int *abort_flag = &sh.abort_flag;

    if (threadIdx.x == 0) {
        for (int s = 0; s < PR_STAGES; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);    // used in the even CTA: both CTAs' copies report there
            mbar_init(smem_u32(&sh.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh.tmem_full[b]), 1);
            mbar_init(smem_u32(&sh.tmem_empty[b]), 2 * PR_EPI_WARPS);   // used in the even CTA: the epilogue warps of both
        }
        mbar_init(smem_u32(&sh.mma_drain), 1);
        sh.abort_flag = sh.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {   // TMEM: all 512 columns (two 256-column accumulators), in both CTAs
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // both CTAs' barriers exist before either signals the other's
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    grid_dependency();

    const int n_tiles = g.m_tiles * g.n_tiles;
    const int pair = SPLIT ? blockIdx.x / (2 * g.split) : blockIdx.x >> 1, pairs = SPLIT ? n_tiles : gridDim.x >> 1;
    const int all_blocks = (g.k + BK - 1) / BK;
    const int kb0 = SPLIT ? all_blocks * (int)part / g.split : 0;
    const int kblocks = SPLIT ? all_blocks * ((int)part + 1) / g.split - kb0 : all_blocks;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; tile < n_tiles && ok; tile += pairs) {
                int mt, nt;
                pair_tile(g, tile, mt, nt);
                const int x_row = mt * PR_TILE + (int)rank * 128;
                const int w_row = SWIGLU ? (rank ? g.n : 0) + nt * 128 : nt * PR_TILE + (int)rank * 128;
                for (int kb = 0; kb < kblocks; ++kb, ++it) {
                    const int s = it % PR_STAGES;
                    if (!mbar_wait(smem_u32(&sh.empty[s]), ((it / PR_STAGES) & 1) ^ 1, abort_flag, g.wait_limit)) { ok = false; break; }
                    const uint32_t full = map_to_cta(smem_u32(&sh.full[s]), leader);
                    const uint32_t dst = smem_u32(ring + s * PR_STAGE_BYTES);
                    if (rank == 0) mbar_expect_tx(smem_u32(&sh.full[s]), 2 * PR_STAGE_BYTES);
                    tma_load_2d_pair(dst, &map_x, (kb0 + kb) * BK, x_row, full);
                    tma_load_2d_pair(dst + PR_HALF_BYTES, &map_w, (kb0 + kb) * BK, w_row, full);
                }
            }
            // a CTA ends when the stages it filled have been read by the MMAs: nothing of it is in flight then, neither a
            // copy nor a release of a stage (also after an abort, within the limit: copies have long landed by then)
            for (uint32_t j = (it > PR_STAGES ? it - PR_STAGES : 0); j < it; ++j)
                if (!mbar_drain(smem_u32(&sh.empty[j % PR_STAGES]), (j / PR_STAGES) & 1)) {
                    *abort_flag = 1;
                    break;
                }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            constexpr uint32_t idesc = make_idesc_i8(256, PR_TILE);
            uint32_t it = 0, tcount = 0;
            bool ok = true;
            for (int tile = pair; tile < n_tiles && ok; tile += pairs, ++tcount) {
                const int buf = tcount & 1;
                if (!mbar_wait(smem_u32(&sh.tmem_empty[buf]), ((tcount >> 1) & 1) ^ 1, abort_flag, g.wait_limit)) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + buf * PR_TILE;
                for (int kb = 0; kb < kblocks; ++kb, ++it) {
                    const int s = it % PR_STAGES;
                    if (!mbar_wait(smem_u32(&sh.full[s]), (it / PR_STAGES) & 1, abort_flag, g.wait_limit)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a0 = smem_u32(ring + s * PR_STAGE_BYTES);
                    const uint64_t da = make_desc(a0), db = make_desc(a0 + PR_HALF_BYTES);
#pragma unroll
                    for (int k = 0; k < BK / 32; ++k) tc_mma_i8_pair(d_tmem, da + 2 * k, db + 2 * k, idesc, (kb | k) ? 1u : 0u);
                    tc_commit_pair(smem_u32(&sh.empty[s]), pair_mask);
                }
                if (ok) tc_commit_pair(smem_u32(&sh.tmem_full[buf]), pair_mask);
            }
            tc_commit_pair_local(smem_u32(&sh.mma_drain));
            if (!mbar_drain(smem_u32(&sh.mma_drain), 0)) *abort_flag = 1;
        }
    } else if (!SPLIT) {
        // ---------------- epilogue: warp w reads TMEM lanes 32*(w%4) .. +31 = rows of this CTA's half of the tile; the two
        // warps of a quarter take alternate pieces of 64 bytes
        const int q = warp & 3, c_first = warp >= 6 ? 32 : 0;
        unsigned char *stg = stage_base + (warp - 2) * PR_STG_WARP;
        uint32_t tcount = 0;
        bool gave_up = false;   // after an expired wait a warp only keeps the others' barriers
        for (int tile = pair; tile < n_tiles; tile += pairs, ++tcount) {
            const int buf = tcount & 1;
            int mt, nt;
            pair_tile(g, tile, mt, nt);
            const int row0 = mt * PR_TILE + (int)rank * 128 + q * 32;   // token of lane 0
            const int col0 = nt * (SWIGLU ? 128 : PR_TILE);
            // scales come while the tile is still being multiplied; the barrier of the epilogue warps also keeps a buffer
            // from being overwritten while a warp is two tiles behind
            const float xs = row0 + lane < g.T ? g.xs[row0 + lane] : 0.0f;
            const int wc = threadIdx.x - 64, wcol = col0 + (SWIGLU ? wc & 127 : wc);
            sh.ws[buf][wc] = wcol < g.n ? g.ws[wcol + (SWIGLU && wc >= 128 ? g.n : 0)] : 0.0f;
            // (one thread polls, the others wait in hardware: pollers slow the two threads that feed the tensor cores)
            if (threadIdx.x == 64 && !gave_up && !mbar_wait(smem_u32(&sh.tmem_full[buf]), (tcount >> 1) & 1, abort_flag, g.wait_limit)) sh.gave_up = 1;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            gave_up = *(volatile int *)&sh.gave_up != 0;
            if (gave_up) continue;
            tc_fence_after();
            const uint32_t tm = tmem_base + buf * PR_TILE + ((uint32_t)(q * 32) << 16);
            pair_store<SWIGLU>(g, row0, xs, col0, c_first, SWIGLU ? 128 : PR_TILE, sh.ws[buf], stg, lane, [&](int c, auto &v) {
                if constexpr (sizeof(v) == 128) tc_ld32(tm + c, v);
                else tc_ld16(tm + c, v);
            });
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&sh.tmem_empty[buf]), 0));
        }
    } else {
        // ---------------- epilogue of a shared tile: scales, then this pair's sums as [column][128 rows] over the ring:
        // a peer's warp then reads 128 consecutive bytes (rows of 16-byte pieces in the lanes cost it 4 to 8 us more)
        const int q = warp & 3, wc = threadIdx.x - 64;
        int mt, nt;
        pair_tile(g, pair, mt, nt);
        const int wcol = nt * (SWIGLU ? 128 : PR_TILE) + (SWIGLU ? wc & 127 : wc);
        sh.ws[0][wc] = wcol < g.n ? g.ws[wcol + (SWIGLU && wc >= 128 ? g.n : 0)] : 0.0f;
        if (threadIdx.x == 64) mbar_wait(smem_u32(&sh.tmem_full[0]), 0, abort_flag, g.wait_limit);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        tc_fence_after();
        int32_t *sums = reinterpret_cast<int32_t *>(ring) + q * 32 + lane;
        for (int c = warp >= 6 ? 32 : 0; c < PR_TILE; c += 64) {
            uint32_t v[32];
            tc_ld32(tmem_base + c + ((uint32_t)(q * 32) << 16), v);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) sums[(c + j) * 128] = (int32_t)v[j];
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort_flag && g.status) atomicMax(g.status, (int)SPICE_ERR_TIMEOUT);
    cluster_sync();   // the pair's MMAs, copies and signals are over in both CTAs; SPLIT: everybody's sums are there
    if (SPLIT) {
        if (warp >= 2) {
            int mt, nt;
            pair_tile(g, pair, mt, nt);
            const int q = warp & 3, row0 = mt * PR_TILE + (int)rank * 128 + q * 32;
            const float xs = row0 + lane < g.T ? g.xs[row0 + lane] : 0.0f;
            constexpr int PIECES = SWIGLU ? 4 : 8;   // pieces of 32 columns, dealt out to the pairs
            const int first = PIECES * (int)part / g.split * 32, last = PIECES * ((int)part + 1) / g.split * 32;
            const uint32_t at = smem_u32(ring) + (uint32_t)(q * 32 + lane) * 4u;
            pair_store<SWIGLU>(g, row0, xs, nt * (SWIGLU ? 128 : PR_TILE), first + (warp >= 6 ? 32 : 0), last, sh.ws[0],
                               stage_base + (warp - 2) * PR_STG_WARP, lane, [&](int c, auto &v) {
                constexpr int N = sizeof(v) / 4;
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = 0u;
#pragma unroll 2
                for (int r = 0; r < g.split; ++r) {
                    const uint32_t peer = map_to_cta(at + (uint32_t)c * 512u, 2 * (uint32_t)r + rank);
                    uint32_t p[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(p[j]) : "r"(peer + j * 512));
#pragma unroll
                    for (int j = 0; j < N; ++j) v[j] += p[j];
                }
            });
        }
        cluster_sync();   // nobody leaves while a peer reads its sums
    }
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512));
}

// ------------------------------------------------------------------------------------------------ host side
constexpr int PR_MAX_SPLIT = 4;
std::atomic<uint32_t> wait_limit{WAIT_LIMIT};   // (SPICE_OPT_I8_WAIT_LIMIT)

// What a device is asked once: dynamic shared memory limits are raised, and how many clusters of c CTAs run at the same time
// when an SM holds one CTA (a cluster stays inside a group of SMs; clusters beyond that wait for a whole round).
struct DeviceFacts {
    std::atomic<bool> ready;
    int clusters[SK_MAX_SPLIT + 1];
};
static_assert(2 * PR_MAX_SPLIT <= SK_MAX_SPLIT, "the sizes that are asked for");
const DeviceFacts *device_facts(int dev, int sms) {
    static DeviceFacts facts[64];
    static std::mutex mutex;
    DeviceFacts &f = facts[dev];
    if (f.ready.load(std::memory_order_acquire)) return &f;
    std::lock_guard<std::mutex> lock(mutex);
    if (f.ready.load(std::memory_order_relaxed)) return &f;
    auto raise = [](const void *kernel, size_t bytes) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
    };
    if (!raise((const void *)gemm_i8_skinny_kernel<false>, SK_MAX_SMEM) || !raise((const void *)gemm_i8_skinny_kernel<true>, SK_MAX_SMEM) ||
        !raise((const void *)gemm_i8_pair_kernel<false, false>, PR_SMEM) || !raise((const void *)gemm_i8_pair_kernel<true, false>, PR_SMEM) ||
        !raise((const void *)gemm_i8_pair_kernel<false, true>, PR_SMEM) || !raise((const void *)gemm_i8_pair_kernel<true, true>, PR_SMEM))
        return nullptr;
    for (int c = 2; c <= SK_MAX_SPLIT; ++c) {
        cudaLaunchConfig_t lc{};
        lc.gridDim = dim3((unsigned)(c * sms), 1, 1);
        lc.blockDim = dim3(PR_THREADS, 1, 1);
        lc.dynamicSmemBytes = PR_SMEM;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)c;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        lc.attrs = at;
        lc.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&f.clusters[c], gemm_i8_pair_kernel<false, true>, &lc) != cudaSuccess) return nullptr;
    }
    f.ready.store(true, std::memory_order_release);
    return &f;
}

template <int NT, int NW, int UN, bool SWIGLU>
bool launch_few(const GemmI8Args &g, const int8_t *x, const int8_t *w, int blocks, cudaStream_t st) {
    auto *kernel = NT >= 4 || (g.k + 63) / 64 <= NW * UN ? gemm_i8_few_kernel<NT, NW, UN, true, SWIGLU>
                                                          : gemm_i8_few_kernel<NT, NW, UN, (NT >= 4), SWIGLU>;
    return launch_early(kernel, dim3((unsigned)blocks), NW * 32, 0, st, 1, x, w, g);
}

template <bool SWIGLU>
spice_status launch_gemm_i8(GemmI8Args g, const int8_t *x, const int8_t *w, cudaStream_t st) {
    int dev = 0;
    const int sms = current_device_sms(&dev);
    if (sms <= 0) return SPICE_ERR_CUDA;
    const DeviceFacts *facts = device_facts(dev, sms);
    if (!facts) return SPICE_ERR_CUDA;
    const int w_rows = SWIGLU ? 2 * g.n : g.n;
    const int kblocks = (g.k + BK - 1) / BK;
    const int64_t weights = (int64_t)w_rows * g.k;
    // Up to some MB of weights the short start wins, beyond that the reads of the tokens cost more than it saves.
    // 512 x 512, 2048 x 2816, 5632 x 2048, 11264 x 2048, 3584 x 20480, 40960 x 3584 weights, us with this kernel / the
    // tensor-memory one:  8 tokens 1.5/3.6, 3.1/5.7, 4.3/6.8, 7.0/8.7, 17.5/15.9, 25.6/25.9;  16 tokens 1.9/3.7, 4.5/6.0,
    // 4.6/7.1, 7.7/8.8, 20/16, 37/26;  32 tokens 2.2/4.1, 6.7/6.6, 6.0/7.8, 10.3/9.7, 35/17, 46/26
    if ((g.T <= 16 && weights <= (48 << 20)) || (g.T <= FEW_MAX_TOKENS && weights <= (16 << 20))) {
        const int blocks = (g.n + (SWIGLU ? 7 : 15)) / (SWIGLU ? 8 : 16);
        const bool wide = blocks < 2 * sms;   // few blocks: sixteen warps in each, enough bytes in flight
        const bool ok = g.T <= 8 ? (wide ? launch_few<1, 16, 4, SWIGLU>(g, x, w, blocks, st) : launch_few<1, 8, 4, SWIGLU>(g, x, w, blocks, st))
                        : g.T <= 16 ? (wide ? launch_few<2, 16, 4, SWIGLU>(g, x, w, blocks, st) : launch_few<2, 8, 4, SWIGLU>(g, x, w, blocks, st))
                        : launch_few<4, 8, 2, SWIGLU>(g, x, w, blocks, st);
        return ok ? SPICE_OK : SPICE_ERR_CUDA;
    }
    CUtensorMap map_x, map_w;
    g.m_tiles = (g.T + PR_TILE - 1) / PR_TILE;
    g.n_tiles = SWIGLU ? (g.n + 127) / 128 : (g.n + PR_TILE - 1) / PR_TILE;
    if ((int64_t)g.m_tiles * g.n_tiles > 0x3fffffff) return SPICE_ERR_UNSUPPORTED_SHAPE;
    const int tile_n = SWIGLU ? 64 : 128;
    const int row_tiles = (g.n + tile_n - 1) / tile_n;
    // Up to 512 tokens either tensor-memory kernel can be the faster one.  Estimates in ns: a start, what a token column of a
    // tile costs in sums, and the bytes that the CTAs bring in at 11.5 TB/s (narrower token tiles: fewer columns, the weights
    // more often), against a start and 310 ns per 128 of the reduction for every round of the pairs over their tiles.
    // Measured, few-token kernel / pairs, us, in the order above:  64 tokens 3.8/5.3, 6.9/11.1, 8.7/10.2, 10.6/10.8, 18/25,
    // 28/36;  128 tokens 3.9/6.1, 8.0/12.0, 9.9/10.7, 12.7/11.7, 21/25, 33/37;  192 tokens 3.8/6.2, 8.7/12.0, 10.6/10.7,
    // 13.7/11.7, 27/25, 53/38;  256 tokens 4.0/6.2, 9.1/12.1, 12.0/10.8, 15.3/11.9, 29/26, 56/38;  384 tokens 4.4/6.3, 10.3/12.4.
    // (Where the pairs are ahead, the other figure is that of tiles of up to 128 tokens, the widest there are.)
    int64_t few_ns = INT64_MAX;
    int token_tiles = 1;
    for (int tt = (g.T + 127) / 128; g.T <= 512 && tt <= 16; ++tt) {
        const int cols = ((g.T + tt - 1) / tt + 15) & ~15, tiles = row_tiles * tt;
        if ((g.T + cols - 1) / cols < tt) continue;   // (fewer tiles of this width do)
        // the reduction is split as far as all clusters run at once, two CTAs to an SM, with three stages each at least (148 SMs:
        // 148, 90, 66, 52, 44, 30, 30 clusters of 2 to 8)
        int split = max(1, min(SK_MAX_SPLIT, kblocks / 3));
        while (split > 1 && tiles > 2 * facts->clusters[split]) --split;
        const int64_t ns = 4000 + (split > 1 ? 46 : 16) * cols + (int64_t)tiles * kblocks * (SK_W_BYTES + cols * BK) / 11500;
        if (ns < few_ns) {
            few_ns = ns;
            token_tiles = tt;
            g.cols = cols;
            g.split = split;
        }
    }
    const int tiles = row_tiles * token_tiles;
    const int64_t tiles_pair = (int64_t)g.m_tiles * g.n_tiles;
    const int64_t rounds = (tiles_pair + sms / 2 - 1) / (sms / 2);
    int64_t pair_ns = 5200 + rounds * kblocks * 310 + (rounds - 1) * 2000;
    // Fewer tiles than pairs: 2 to 4 pairs share a tile's reduction, as long as all the clusters run at once (512 x 3584 x
    // 20480 with one / two pairs to a tile: 54.6 / 33.8 us, 256 x 3584 x 20480 with one / four: 54 / 25.5).
    int share = 1;
    for (int s = 2; s <= PR_MAX_SPLIT; ++s) {
        const int64_t ns = 9000 + (s - 2) * 1850 + (int64_t)((kblocks + s - 1) / s) * 310;
        if (tiles_pair <= facts->clusters[2 * s] && kblocks >= 2 * s && ns < pair_ns) {
            pair_ns = ns;
            share = s;
        }
    }
    if (few_ns <= pair_ns) {
        int per_sm = (tiles * g.split + sms - 1) / sms;
        per_sm = std::max(g.split > 1 ? 2 : 1, std::min(per_sm, 3));   // (clusters pack badly with one CTA per SM)
        const int per_cta = (kblocks + g.split - 1) / g.split;
        const int stage_bytes = SK_W_BYTES + g.cols * BK;
        g.stages = max(1, min(min(per_cta, SK_MAX_STAGES), (228 / per_sm - 4) * 1024 / stage_bytes));
        const size_t red = (size_t)min(g.cols, g.T) * 512;
        // A CTA takes at least the share of shared memory that it takes of TMEM (512 columns against 228 KB with the 1 KB
        // the system adds): however the CTAs of calls on different streams mix on an SM, no TMEM allocation has to wait,
        // and a cluster never holds columns that a CTA of another cluster needs to reach its own barrier.
        int tmem_cols = 32;
        while (tmem_cols < g.cols) tmem_cols *= 2;
        const size_t smem = std::max({(size_t)g.stages * stage_bytes + 1024, red + 1024, (size_t)(456 * tmem_cols - 1024)});
        if (!tc_encode_map2_bytes(&map_w, w, (uint64_t)w_rows, (uint64_t)g.k, tile_n) ||
            !tc_encode_map2_bytes(&map_x, x, (uint64_t)g.T, (uint64_t)g.k, (uint32_t)g.cols))
            return SPICE_ERR_CUDA;
        return launch_early(gemm_i8_skinny_kernel<SWIGLU>, dim3((unsigned)(row_tiles * g.split), (unsigned)token_tiles, 1), SK_THREADS, smem,
                            st, g.split, map_w, map_x, g) ? SPICE_OK : SPICE_ERR_CUDA;
    }
    if (!tc_encode_map2_bytes(&map_x, x, (uint64_t)g.T, (uint64_t)g.k, 128) ||
        !tc_encode_map2_bytes(&map_w, w, (uint64_t)w_rows, (uint64_t)g.k, 128))
        return SPICE_ERR_CUDA;
    bool ok;
    if (share > 1) {
        g.split = share;
        ok = launch_early(gemm_i8_pair_kernel<SWIGLU, true>, dim3((unsigned)(2 * share * tiles_pair)), PR_THREADS, PR_SMEM, st, 2 * share,
                          map_x, map_w, g);
    } else {
        const int pairs = max(1, min(sms / 2, g.m_tiles * g.n_tiles));
        ok = launch_early(gemm_i8_pair_kernel<SWIGLU, false>, dim3(2 * (unsigned)pairs), PR_THREADS, PR_SMEM, st, 2, map_x, map_w, g);
    }
    return ok ? SPICE_OK : SPICE_ERR_CUDA;
}

template <bool SWIGLU>
spice_status call_gemm_i8(const int8_t *x_q, const float *x_scale, const int8_t *w_q, const float *w_scale, int32_t T, int32_t n,
                          int32_t k, int32_t out, void *y, int32_t *device_status, void *stream) {
    if (T < 0 || n < 8 || n % 8 || k < 16 || k % 16 ||
        (out != SPICE_OUT_BF16 && out != SPICE_OUT_F32 && out != SPICE_OUT_F32_ADD))
        return SPICE_ERR_INVALID_ARG;
    if (k > MAX_K || n > (1 << 24) || T > (1 << 24)) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    if (!x_q || !x_scale || !w_q || !w_scale || !y || !aligned16(x_q) || !aligned16(w_q) || !aligned16(w_scale) || !aligned16(y) ||
        (reinterpret_cast<uintptr_t>(x_scale) & 3u) || (reinterpret_cast<uintptr_t>(device_status) & 3u))
        return SPICE_ERR_INVALID_ARG;
    GemmI8Args g{};
    g.xs = x_scale;
    g.ws = w_scale;
    g.y = y;
    g.T = T;
    g.n = n;
    g.k = k;
    g.out = out;
    g.status = device_status;
    g.wait_limit = wait_limit.load(std::memory_order_relaxed);
    return launch_gemm_i8<SWIGLU>(g, x_q, w_q, static_cast<cudaStream_t>(stream));
}

}  // namespace

void set_gemm_i8_wait_limit(uint32_t polls) { wait_limit.store(polls, std::memory_order_relaxed); }

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_gemm_i8(const int8_t *x_q, const float *x_scale, const int8_t *w_q, const float *w_scale, int32_t T,
                                      int32_t n, int32_t k, int32_t out, void *y, int32_t *device_status, void *stream) {
    Range range_("spice_gemm_i8");
    return call_gemm_i8<false>(x_q, x_scale, w_q, w_scale, T, n, k, out, y, device_status, stream);
}

extern "C" spice_status spice_swiglu_i8(const int8_t *x_q, const float *x_scale, const int8_t *w_gate_up_q, const float *w_scale,
                                        int32_t T, int32_t inter, int32_t k, spice_bf16 *act, int32_t *device_status, void *stream) {
    Range range_("spice_swiglu_i8");
    return call_gemm_i8<true>(x_q, x_scale, w_gate_up_q, w_scale, T, inter, k, SPICE_OUT_BF16, act, device_status, stream);
}
