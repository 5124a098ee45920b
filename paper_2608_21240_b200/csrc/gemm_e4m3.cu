// Products of 8-bit floating-point rows with a scale for each block of 128, dense or over rows sorted by expert:
//
//   y[t, j] = sum_b xs[t,b] ws[j/128, b] sum_{i in block b} x[t,i] w[j,i]            (bf16, fp32, or added to fp32)
//   SwiGLU:   g, u = the products with the gate and the up rows;  a = g / (1 + e^-g) u;  codes and scales of a in blocks of 128
//
// with the weights of group g for the rows offset[g] .. offset[g+1].  The inner sums are 128 products of E4M3 values, exact
// in the tensor cores' operands and added in their fp32 accumulators; every block's sum is multiplied by its two scales and
// added in fp32 registers, so no scale is rounded into an operand and long reductions are sums of fp32 sums.
//
// Three kernels.  Few rows a group: every weight byte is used for few products and the call is bound by streaming the weights,
// through a ring in shared memory into warp-wide products.  A few tokens and few weights: neither ring nor clusters, whose start
// and sums would cost more than the call.  Otherwise pairs of CTAs (cta_group::2) work on tiles of 256 tokens x 256 weight rows,
// persistent.
#include <cuda_fp8.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

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
    uint32_t most_tiles;     // tiles of a call, at most: groups that overlap can have more of them than an index holds
    int32_t split;           // some rows a group: CTAs of a cluster that share a reduction
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
// four neighbouring columns
__device__ __forceinline__ void store4(const GemmE4m3Args &g, size_t at, float4 v) {
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
__device__ __forceinline__ void store1(const GemmE4m3Args &g, size_t at, float v) {
    if (g.out == SPICE_OUT_BF16) static_cast<__nv_bfloat16 *>(g.y)[at] = __float2bfloat16_rn(v);
    else if (g.out == SPICE_OUT_F32) static_cast<float *>(g.y)[at] = v;
    else static_cast<float *>(g.y)[at] += v;
}

// ------------------------------------------------------------------------------------------------ few rows a group
// The weights stream through a ring in shared memory at the rate of HBM, and eight warps multiply them with up to 32 tokens in
// warp-wide products: a warp has 32 weight rows (SwiGLU: 16 gate rows and their up rows) and all the tokens, so that only a stage's
// operands pass through shared memory and no sums do.  (In the pair kernel below, whose two accumulators let two blocks be on their way, the
// sums of a block take 0.47 us through tensor memory and back, more than a block of weights takes to arrive.  That is a latency:
// narrower accumulators, with the tokens as the N operand, could have more of them in flight.  Not built.)  Persistent over (group, 256 weight rows, up to 32
// tokens); where those are fewer than the SMs, the CTAs of a cluster share the reduction of one and add up through distributed
// shared memory.  96 rows over 64 groups: SwiGLU 1408 x 2048 59 us, 0.89 of the measured copy rate; product 2048 x 1408 33 us, 0.80.
// From 16 tokens on the products of a block (400 a cycle and SM) take longer than its weights: 3584 x 20480 with 1 / 16 / 32 tokens
// 15.7 / 18.5 / 27.6 us.
constexpr int ST_WARPS = 8, ST_THREADS = ST_WARPS * 32 + 32, ST_MAX_SPLIT = 8;
constexpr int ST_W_BYTES = 256 * BK;
constexpr int ST_RED_PITCH = 260;                 // fp32 sums of a token's 256 weight rows, padded against bank conflicts

template <int NT>
struct StreamShape {
    static constexpr int TOKENS = NT * 8, STAGE_BYTES = ST_W_BYTES + TOKENS * BK, STAGES = 6;
};
template <int NT>
struct StreamShared {
    float xs[StreamShape<NT>::STAGES][StreamShape<NT>::TOKENS];
    float peak[ST_WARPS][StreamShape<NT>::TOKENS];    // SwiGLU: largest magnitude of a token's columns, per warp
    int32_t first[MAX_GROUPS + 1];                    // tiles before each group
    alignas(8) unsigned long long full[6], empty[6];
    int abort_flag;
};
template <int NT>
constexpr size_t stream_smem() {
    return sizeof(StreamShared<NT>) + (size_t)StreamShape<NT>::STAGES * StreamShape<NT>::STAGE_BYTES + 1024;
}
static_assert(stream_smem<4>() <= 232448, "what a block can have");
static_assert(32 * ST_RED_PITCH * 4 <= 6 * ST_W_BYTES, "the sums fit in the ring");

// Tiles before each group, by one warp: per group (its rows / `rows`, rounded up) x n_tiles; a group whose offsets are not in
// order or out of range has none.  Sums stop at g.most_tiles, which is 2^30 at most: only groups that overlap get there (512 of
// 1024 groups with all rows each, say), and what is behind it is left out.
__device__ __forceinline__ void count_tiles(const GemmE4m3Args &g, int rows, int32_t *first) {
    const int lane = threadIdx.x & 31;
    uint32_t carry = 0;
    for (int base = 0; base < g.G; base += 32) {
        const int i = base + lane;
        int b = 0, e = g.T;
        uint32_t tiles = 0;
        if (i < g.G && g.offset) {
            b = load_s32(g.offset + i);
            e = load_s32(g.offset + i + 1);
        }
        if (i < g.G) {
            if (b < 0 || e < b || e > g.T) {
                if (blockIdx.x == 0 && g.status) atomicMax(g.status, (int)SPICE_ERR_BAD_TABLE);
            } else {
                tiles = (e - b + rows - 1) / rows * g.n_tiles;
            }
        }
        uint32_t incl = min(tiles, g.most_tiles);
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl = min(incl + v, g.most_tiles);
        }
        incl = min(incl + carry, g.most_tiles);
        if (i < g.G) first[i + 1] = (int)incl;
        carry = __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) first[0] = 0;
}

struct Tile {
    int group, t0, rows, nt;   // first token, tokens, weight tile
};

__device__ __forceinline__ void mma_e4m3(float (&d)[4], int a0, int a1, int a2, int a3, int b0, int b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr));
}

// A token whose sums lie in the shared memory of several CTAs of the cluster, part p in CTA p * step + base at the address `at`: 256
// weight rows (SwiGLU: 128 gate rows and their up rows).  By a warp: its lanes have four neighbouring rows each, and all parts of them
// (up to four) are on their way at once.
template <bool SWIGLU>
__device__ __forceinline__ void finish_token(const GemmE4m3Args &g, uint32_t at, int parts, int step, int base, size_t token, int nt, bool ok, int lane) {
    float4 v[2];
    v[0] = v[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int p0 = 0; p0 < parts; p0 += 4) {
        float4 o[4][2];
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                o[p][z] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (p0 + p < parts)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(o[p][z].x), "=f"(o[p][z].y), "=f"(o[p][z].z), "=f"(o[p][z].w)
                                 : "r"(map_to_cta(at + z * 512 + lane * 16, (uint32_t)((p0 + p) * step + base))));
            }
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int z = 0; z < 2; ++z) v[z] = make_float4(v[z].x + o[p][z].x, v[z].y + o[p][z].y, v[z].z + o[p][z].z, v[z].w + o[p][z].w);
    }
    if constexpr (SWIGLU) {
        const float a[4] = {silu_times(v[0].x, v[1].x), silu_times(v[0].y, v[1].y), silu_times(v[0].z, v[1].z), silu_times(v[0].w, v[1].w)};
        float big = max_magnitude(max_magnitude(max_magnitude(fabsf(a[0]), a[1]), a[2]), a[3]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) big = max_magnitude(big, __shfl_xor_sync(0xffffffffu, big, o));
        const OutScale q(big);
        if (ok) {
            *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(g.y) + token * g.n + nt * 128 + lane * 4) =
                code2(a[0], a[1], q.r) | code2(a[2], a[3], q.r) << 16;
            if (lane == 0) g.ys[token * (g.n / 128) + nt] = q.scale;
        }
    } else if (ok) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const int col = nt * 256 + z * 128 + lane * 4;
            if (col < g.n) store4(g, token * g.n + col, v[z]);
        }
    }
}

template <int NT, bool SWIGLU, bool SPLIT>
__global__ void __launch_bounds__(ST_THREADS, 1)
    gemm_e4m3_stream_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const GemmE4m3Args g) {
    using Shape = StreamShape<NT>;
    constexpr uint32_t STAGES = Shape::STAGES;
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    StreamShared<NT> &sh = *reinterpret_cast<StreamShared<NT> *>(ring + STAGES * Shape::STAGE_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh.abort_flag;
    const int split = SPLIT ? g.split : 1, rank = SPLIT ? (int)cluster_rank() : 0;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 33);           // the copies, and the scales that a warp fetches
            mbar_init(smem_u32(&sh.empty[s]), ST_WARPS);
        }
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    grid_dependency();
    if (warp == ST_WARPS) count_tiles(g, Shape::TOKENS, sh.first);
    __syncthreads();
    const int n_items = sh.first[g.G];
    const int team = blockIdx.x / split, teams = gridDim.x / split;
    const int kb0 = g.kb * rank / split, kbs = g.kb * (rank + 1) / split - kb0;
    const uint32_t ring0 = smem_u32(ring), full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
    auto find = [&](int item, int &group) {
        while (item >= sh.first[group + 1]) ++group;
        const int begin = g.offset ? load_s32(g.offset + group) : 0, m = (g.offset ? load_s32(g.offset + group + 1) : g.T) - begin;
        const int parts = (m + Shape::TOKENS - 1) / Shape::TOKENS, in = item - sh.first[group];
        const int t0 = in % parts * Shape::TOKENS;
        return Tile{group, begin + t0, min(Shape::TOKENS, m - t0), in / parts};
    };

    if (warp == ST_WARPS) {
        uint32_t s = 0, phase = 1, filled = 0, limit = g.wait_limit;
        int group = 0;
        auto land = [&]() {   // everything that was ordered has landed
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (lane == 0)
                for (uint32_t left = filled; left > 0; --left) {
                    const uint32_t back = s >= left ? 0u : 1u;   // the stage filled `left` blocks ago: in this round of the ring, or the one before
                    if (!mbar_drain(full0 + (s + back * STAGES - left) * 8, phase ^ 1 ^ back)) {
                        *abort_flag = 1;
                        break;
                    }
                }
            __syncwarp();
        };
        for (int item = team; item < n_items && (SPLIT || limit != 0); item += teams) {
            const Tile t = find(item, group);
            const int w0 = SWIGLU ? 2 * t.group * g.n + t.nt * 128 : t.group * g.n + t.nt * 256, w1 = SWIGLU ? w0 + g.n : w0 + 128;
            for (int b = kb0; b < kb0 + kbs; ++b) {
                mbar_wait_quick(empty0 + s * 8, phase, abort_flag, limit);
                if (limit == 0) break;
                const uint32_t dst = ring0 + s * Shape::STAGE_BYTES, full = full0 + s * 8;
                if (lane == 0) {
                    mbar_expect_tx(full, Shape::STAGE_BYTES);
                    tma_load_2d(dst, &map_w, b * BK, w0, full);
                    tma_load_2d(dst + ST_W_BYTES / 2, &map_w, b * BK, w1, full);
                    tma_load_2d(dst + ST_W_BYTES, &map_x, b * BK, t.t0, full);
                }
#pragma unroll
                for (int c = lane; c < Shape::TOKENS; c += 32) {   // (of tokens that are not there: zeros)
                    const float *from = g.xs + (size_t)(t.t0 + min(c, t.rows - 1)) * g.kb + b;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(&sh.xs[s][c])), "l"(from), "r"(c < t.rows ? 4 : 0) : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full) : "memory");
                filled = min(filled + 1, STAGES);
                if (++s == STAGES) {
                    s = 0;
                    phase ^= 1;
                }
            }
            if (SPLIT) {   // the sums lie in the ring between these two: the next item is ordered behind them
                land();
                filled = 0;
                cluster_sync();
                cluster_sync();
            }
        }
        if (!SPLIT) land();   // before the CTA ends
    } else {
        const int r4 = lane >> 2, c2 = 2 * (lane & 3);
        const int row_blocks = ((SWIGLU ? 2 * g.n : g.n) + 127) / 128;
        // rows of this warp in a stage: its two tiles of 16
        const int wr0 = SWIGLU ? warp * 16 : warp * 32, wr1 = SWIGLU ? 128 + warp * 16 : warp * 32 + 16;
        // lane's row and 16-byte piece in a load of four 8 x 16 byte matrices (A: rows 0-7, 8-15, then the next 16 bytes; B: 16 bytes
        // after 16 bytes); rows of 128 bytes, pieces swizzled by the row
        const int ar = (lane & 7) + (lane & 8), ac = lane >> 4, br = lane & 7, bc = lane >> 3;
        uint32_t s = 0, phase = 0, limit = g.wait_limit;
        int group = 0;
        for (int item = team; item < n_items; item += teams) {
            const Tile t = find(item, group);
            const int nb = SWIGLU ? t.nt : min(t.nt * 2 + warp / 4, row_blocks - 1);
            const float *ws = g.ws + ((size_t)t.group * row_blocks + nb) * g.kb + kb0, *wu = ws + (size_t)(g.n / 128) * g.kb;
            float acc[2][NT][4];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[r][i][j] = 0.0f;
            float w_next = load_f32(ws), u_next = SWIGLU ? load_f32(wu) : 0.0f;
#pragma unroll 1
            for (int b = 0; b < kbs; ++b) {
                const float sw[2] = {w_next, SWIGLU ? u_next : w_next};
                const int ahead = min(b + 1, kbs - 1);
                w_next = load_f32(ws + ahead);
                if (SWIGLU) u_next = load_f32(wu + ahead);
                mbar_wait_quick(full0 + s * 8, phase, abort_flag, limit);
                const uint32_t wt = ring0 + s * Shape::STAGE_BYTES, xt = wt + ST_W_BYTES + br * BK;
                uint32_t a[2][4][4];
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) ldmatrix4(wt + ((r ? wr1 : wr0) + ar) * BK + (((2 * k + ac) ^ (ar & 7)) << 4), a[r][k]);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    uint32_t lo[4], hi[4];
                    ldmatrix4(xt + i * 8 * BK + ((bc ^ br) << 4), lo);
                    ldmatrix4(xt + i * 8 * BK + (((4 + bc) ^ br) << 4), hi);
                    const float2 sx = *reinterpret_cast<const float2 *>(&sh.xs[s][i * 8 + c2]);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_e4m3(d, a[r][0][0], a[r][0][1], a[r][0][2], a[r][0][3], lo[0], lo[1]);
                        mma_e4m3(d, a[r][1][0], a[r][1][1], a[r][1][2], a[r][1][3], lo[2], lo[3]);
                        mma_e4m3(d, a[r][2][0], a[r][2][1], a[r][2][2], a[r][2][3], hi[0], hi[1]);
                        mma_e4m3(d, a[r][3][0], a[r][3][1], a[r][3][2], a[r][3][3], hi[2], hi[3]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[r][i][j] = fmaf(d[j], (j & 1 ? sx.y : sx.x) * sw[r], acc[r][i][j]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(empty0 + s * 8);
                if (++s == STAGES) {
                    s = 0;
                    phase ^= 1;
                }
            }
            const bool ok = limit != 0;
            if constexpr (SPLIT) {
                // ---- sums as [token][256 weight rows] over the ring, which is filled again behind the second barrier only.  A cluster has
                // one item; where groups overlap there are more items than clusters.  Every warp of every CTA passes two cluster barriers
                // per item, also after an expired wait, and all CTAs of a cluster count the same items: none waits for an arrival that
                // does not come.
                asm volatile("bar.sync 1, 256;" ::: "memory");   // (all have read their last stage)
                float *red = reinterpret_cast<float *>(ring);
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) red[(i * 8 + c2 + (j & 1)) * ST_RED_PITCH + (r ? wr1 : wr0) + r4 + (j >> 1) * 8] = acc[r][i][j];
                cluster_sync();
                // every CTA finishes some of the tokens, a warp a token at a time
                for (int c = rank + warp * split; c < t.rows; c += ST_WARPS * split)
                    finish_token<SWIGLU>(g, smem_u32(red + c * ST_RED_PITCH), split, 1, 0, (size_t)(t.t0 + c), t.nt, ok, lane);
                if (item + teams < n_items) fence_proxy_async();   // (copies will write where the sums were)
                cluster_sync();   // nobody leaves, or fills the ring, while a peer reads its sums
            } else if constexpr (SWIGLU) {
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    float big[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[0][i][j] = silu_times(acc[0][i][j], acc[1][i][j]);
                        big[j & 1] = max_magnitude(big[j & 1], acc[0][i][j]);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int o = 4; o < 32; o *= 2) big[j] = max_magnitude(big[j], __shfl_xor_sync(0xffffffffu, big[j], o));
                        if (lane < 4) sh.peak[warp][i * 8 + c2 + j] = big[j];
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int c = i * 8 + c2 + j;
                        if (i * 8 >= t.rows) break;
                        float big = sh.peak[0][c];
#pragma unroll
                        for (int p = 1; p < ST_WARPS; ++p) big = max_magnitude(big, sh.peak[p][c]);
                        const OutScale q(big);
                        if (ok && c < t.rows) {
                            uint8_t *to = static_cast<uint8_t *>(g.y) + (size_t)(t.t0 + c) * g.n + t.nt * 128 + warp * 16 + r4;
                            const uint32_t two = code2(acc[0][i][j], acc[0][i][j + 2], q.r);
                            to[0] = (uint8_t)two;
                            to[8] = (uint8_t)(two >> 8);
                            if (warp == 0 && r4 == 0) g.ys[(size_t)(t.t0 + c) * (g.n / 128) + t.nt] = q.scale;
                        }
                    }
                asm volatile("bar.sync 1, 256;" ::: "memory");   // (all have read the magnitudes)
            } else if (ok) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int c = i * 8 + c2 + (j & 1), col = t.nt * 256 + (r ? wr1 : wr0) + r4 + (j >> 1) * 8;
                            if (c < t.rows && col < g.n) store1(g, (size_t)(t.t0 + c) * g.n + col, acc[r][i][j]);
                        }
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort_flag && g.status) atomicMax(g.status, (int)SPICE_ERR_TIMEOUT);
}

// ------------------------------------------------------------------------------------------------ a few tokens and few weights
// A block multiplies 16 weight rows with the rows of one group (eight at most); a warp has two blocks of the reduction, straight from
// global memory.  Both operands are read in pieces of 16 bytes, so the order of the reduction inside a 64-byte piece is the same for
// both and does not matter.  Bound by launch and memory latency: all loads of a call are on their way at once.
constexpr int FEW_WARPS = 8, FEW_TOKENS = 8, FEW_BLOCKS = 2;

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

// The slot-th group that has a row which no group before it has: its number, or -1; groups whose offsets are not in order or out
// of range have no rows.  There are no more of these groups than rows, so a block for each row is enough; all rows of a group that is
// passed over belong to others too.  Groups overlap only behind offsets that fall.
__device__ __forceinline__ int find_group(const GemmE4m3Args &g, int slot, const int32_t *off) {
    const int lane = threadIdx.x & 31;
    uint32_t taken = 0;   // rows of the groups before, a bit each
    bool falls = false;
    for (int base = 0, seen = 0; base < g.G; base += 32) {
        const int i = base + lane, b = i < g.G ? off[i] : 0, e = i < g.G ? off[i + 1] : 0;
        uint32_t own = b >= 0 && e > b && e <= g.T ? (1u << e) - (1u << b) : 0u;
        falls = falls || __any_sync(0xffffffffu, e < b);
        const uint32_t all = taken | __reduce_or_sync(0xffffffffu, own);
        if (falls) {
            uint32_t before = own;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before |= v;
            }
            before = __shfl_up_sync(0xffffffffu, before, 1);
            own &= ~(taken | (lane > 0 ? before : 0u));
        }
        taken = all;
        uint32_t mask = __ballot_sync(0xffffffffu, own != 0);
        const int here = __popc(mask);
        if (seen + here > slot) {
            for (int s = slot - seen; s > 0; --s) mask &= mask - 1;
            return base + __ffs(mask) - 1;
        }
        seen += here;
    }
    return -1;
}

__global__ void __launch_bounds__(FEW_WARPS * 32) gemm_e4m3_few_kernel(const uint8_t *x, const uint8_t *w, const GemmE4m3Args g) {
    __shared__ float red[FEW_WARPS][FEW_TOKENS][20];   // (16, padded: the rows of a warp's store fall into different banks)
    __shared__ int32_t off[MAX_GROUPS + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r8 = lane >> 2, c = lane & 3;
    const int n0 = blockIdx.x * 16;
    grid_dependency();
    if (g.offset) {
        for (int i = threadIdx.x; i <= g.G; i += FEW_WARPS * 32) off[i] = load_s32(g.offset + i);
        __syncthreads();
        if (g.status && blockIdx.x == 0 && blockIdx.y == 0)
            for (int i = threadIdx.x; i < g.G; i += FEW_WARPS * 32)
                if (off[i] < 0 || off[i + 1] < off[i] || off[i + 1] > g.T) atomicMax(g.status, (int)SPICE_ERR_BAD_TABLE);
    }
    // (a loop over more groups than a block for each row costs registers, and 12 for 9 us)
    const int group = g.offset ? find_group(g, blockIdx.y, off) : 0;
    if (group < 0) return;
    const int begin = g.offset ? off[group] : 0, rows = g.offset ? off[group + 1] - begin : g.T;
    const int nv = g.k >> 4, row_blocks = (g.n + 127) / 128;
    const int4 *wr[2], *xr = reinterpret_cast<const int4 *>(x) + (size_t)(begin + r8) * nv;
#pragma unroll
    for (int h = 0; h < 2; ++h)   // (n is a multiple of 8)
        wr[h] = reinterpret_cast<const int4 *>(w) + ((size_t)group * g.n + n0 + r8 + (n0 + 8 * h < g.n ? 8 * h : 0)) * nv;
    const float *ws = g.ws + ((size_t)group * row_blocks + n0 / 128) * g.kb, *xs = g.xs + (size_t)begin * g.kb;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int4 zero = make_int4(0, 0, 0, 0);
    int4 a[FEW_BLOCKS][2][2], bx[FEW_BLOCKS][2];
    float sx[FEW_BLOCKS][2], sw[FEW_BLOCKS];
#pragma unroll
    for (int u = 0; u < FEW_BLOCKS; ++u) {
        const int b = warp + u * FEW_WARPS;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int v = b * 8 + p * 4 + c;
            const bool in = v < nv;
#pragma unroll
            for (int h = 0; h < 2; ++h) a[u][p][h] = in ? load_once(wr[h] + v) : zero;
        }
    }
#pragma unroll
    for (int u = 0; u < FEW_BLOCKS; ++u) {
        const int b = warp + u * FEW_WARPS;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int v = b * 8 + p * 4 + c;
            bx[u][p] = v < nv && r8 < rows ? load_again(xr + v) : zero;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) sx[u][j] = b < g.kb && 2 * c + j < rows ? load_f32(xs + (size_t)(2 * c + j) * g.kb + b) : 0.0f;
        sw[u] = b < g.kb ? load_f32(ws + b) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < FEW_BLOCKS; ++u) {
        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int4 a0 = a[u][p][0], a1 = a[u][p][1], bb = bx[u][p];
            mma_e4m3(d, a0.x, a1.x, a0.y, a1.y, bb.x, bb.y);
            mma_e4m3(d, a0.z, a1.z, a0.w, a1.w, bb.z, bb.w);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(d[j], sx[u][j & 1] * sw[u], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) red[warp][2 * c + (j & 1)][r8 + 8 * (j >> 1)] = acc[j];
    __syncthreads();
    const int t = threadIdx.x / 16, r = threadIdx.x % 16;
    if (t < rows && n0 + r < g.n) {
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < FEW_WARPS; ++q) v += red[q][t][r];
        store1(g, (size_t)(begin + t) * g.n + n0 + r, v);
    }
}

// ------------------------------------------------------------------------------------------------ more rows
constexpr int PR_THREADS = 384, PR_EPI_WARPS = 8;
constexpr uint32_t PR_STAGES = 4;                 // (six are no faster)
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
constexpr int PR_OUT_WARP = 32 * 256;             // an epilogue warp's results on their way out: two boxes of 32 rows x 128 bytes
// All the shared memory there is: a CTA of another kernel beside this one, which holds all of tensor memory, could wait for columns
// that the CTAs of its own cluster need to reach their barriers, on either side.
constexpr size_t PR_SMEM_BYTES = 232448;
static_assert(sizeof(PairShared) + (size_t)PR_STAGES * PR_STAGE_BYTES + PR_EPI_WARPS * PR_OUT_WARP + 1024 <= PR_SMEM_BYTES, "what a block can have");
static_assert(128 * ST_RED_PITCH * 4 <= PR_STAGES * PR_STAGE_BYTES + PR_EPI_WARPS * PR_OUT_WARP, "the sums of a shared tile fit before PairShared");

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

// A block of the reduction is 128 x 128 values of both operands per CTA; its 256 x 256 sums come back from tensor memory, are scaled
// and added in registers, a token per thread, while the other accumulator is multiplied into.  24576 rows over 64 groups of very
// different sizes: product 2048 x 1408 101 to 105 us, SwiGLU 1408 x 2048 199 to 206 us (1400 TFLOP/s), 22 % of the multiplied rows being padding of the last
// tile of a group; the copies alone take 72 and 128 us, the matrix instructions 41 and 91.  With half accumulators (four of 128
// columns) 111 and 203, with 16 epilogue warps 131 and 242.
// SPLIT: the reduction of a tile is shared by the g.split pairs of a cluster (one tile per cluster, one group): each pair leaves its
// sums in its shared memory and finishes its share of the tokens with those of the others.
template <bool SWIGLU, bool SPLIT>
__global__ void __launch_bounds__(PR_THREADS, 1)
    gemm_e4m3_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x128,
                          const __grid_constant__ CUtensorMap map_x16, const __grid_constant__ CUtensorMap map_y, const GemmE4m3Args g) {
    extern __shared__ __align__(16) unsigned char smem_raw[];   // (aligned to 1024 by hand: the swizzled tiles)
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char *out = ring + PR_STAGES * PR_STAGE_BYTES;
    PairShared &sh = *reinterpret_cast<PairShared *>(out + PR_EPI_WARPS * PR_OUT_WARP);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(cluster_rank() & 1u), part = SPLIT ? (int)(cluster_rank() >> 1) : 0;
    const uint32_t leader = 2 * part, pair_mask = 3u << leader;
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
    if (warp == 2) count_tiles(g, PR_TILE, sh.first);
    tc_fence_before();
    __syncthreads();
    cluster_sync();   // both CTAs' barriers exist before either signals the other's
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    const int n_tiles = sh.first[g.G];
    const int pair = SPLIT ? blockIdx.x / (2 * g.split) : blockIdx.x >> 1, pairs = SPLIT ? n_tiles : gridDim.x >> 1;
    const int kb_first = SPLIT ? g.kb * part / g.split : 0, kb_last = SPLIT ? g.kb * (part + 1) / g.split : g.kb;

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
                for (int k0 = kb_first * BK; k0 < kb_last * BK; k0 += BK) {
                    mbar_wait_quick(empty0 + s * 8, phase, abort_flag, limit);
                    if (limit == 0) break;
                    const uint32_t full = map_to_cta(full0 + s * 8, leader), dst = smem_u32(ring) + s * PR_STAGE_BYTES;
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
            const uint32_t total = (uint32_t)(n_tiles > pair ? (n_tiles - pair + pairs - 1) / pairs : 0) * (uint32_t)(kb_last - kb_first);
            for (uint32_t left = (total + 1 - buf) / 2; left > 0; --left) {
                mbar_wait_quick(tmem_empty, tmem_phase, abort_flag, limit);
                mbar_wait_quick(full0 + s * 8, phase, abort_flag, limit);
                if (limit == 0) break;
                tc_fence_after();
                const uint64_t da = desc0 + s * (PR_STAGE_BYTES >> 4), db = da + (PR_HALF_BYTES >> 4);
#pragma unroll
                for (int k = 0; k < BK / 32; ++k) tc_mma_f8_pair(d_tmem, da + 2 * k, db + 2 * k, idesc, k ? 1u : 0u);
                tc_commit_pair(empty0 + s * 8, pair_mask);
                tc_commit_pair(tmem_full, pair_mask);
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
        const uint32_t full0 = smem_u32(&sh.tmem_full[0]), empty0 = map_to_cta(smem_u32(&sh.tmem_empty[0]), leader);
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
            float x = load_f32(xs + kb_first), w = load_f32(ws + kb_first), u = SWIGLU ? load_f32(wu + kb_first) : 0.0f;   // a block ahead
#pragma unroll 1
            for (int kb = kb_first; kb < kb_last; ++kb, ++it) {
                const uint32_t buf = it & 1, tm = tm0 + buf * PR_TILE;
                const float sw = x * w, su = SWIGLU ? x * u : sw;
                const int ahead = min(kb + 1, kb_last - 1);
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
                        tc_pin16(v);
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
            if constexpr (SPLIT) {
                // sums as [128 tokens][256 weight rows] over the ring and what follows it (the last products are over)
                float *sums = reinterpret_cast<float *>(ring) + (q * 32 + lane) * ST_RED_PITCH;
#pragma unroll
                for (int i = 0; i < 64; i += 2)
                    *reinterpret_cast<float4 *>(sums + 2 * i + (SWIGLU ? h * 64 + (i >= 32 ? 64 : 0) : h * 128)) =
                        make_float4(low(acc[i]), high(acc[i]), low(acc[i + 1]), high(acc[i + 1]));
                continue;
            }
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
            } else if (limit != 0 && rows >= 32 && g.out != SPICE_OUT_F32_ADD) {
                // 32 whole rows go out by copies from shared memory, 128 bytes of them at a time (rows of 128 bytes, pieces swizzled
                // by the row), while the next tile is multiplied: stored by the threads themselves a tile's end took 1.5 us longer
                const int col0 = t.nt * PR_TILE + h * 128, size = g.out == SPICE_OUT_BF16 ? 2 : 4;
                const uint32_t to = smem_u32(out) + (uint32_t)(warp - 4) * PR_OUT_WARP, at = to + lane * 128;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    if (g.out == SPICE_OUT_BF16 && z) break;     // (fp32: half of the columns at a time)
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            uint32_t v[4];
                            if (g.out == SPICE_OUT_BF16) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = pack2(low(acc[b * 32 + k * 4 + i]), high(acc[b * 32 + k * 4 + i]));
                            } else {
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const uint64_t a = acc[z * 32 + b * 16 + k * 2 + i];
                                    v[2 * i] = (uint32_t)a;
                                    v[2 * i + 1] = (uint32_t)(a >> 32);
                                }
                            }
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + b * 4096 + ((uint32_t)(k ^ (lane & 7)) << 4)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                        }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        const int x0 = col0 * size + z * 256;
                        for (int b = 0; b < 2; ++b)
                            if (x0 + b * 128 < g.n * size)
                                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                             ::"l"(reinterpret_cast<uint64_t>(&map_y)), "r"(x0 + b * 128), "r"(row), "r"(to + b * 4096) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
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
    if (warp >= 4 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // (results on their way out)
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort_flag && g.status) atomicMax(g.status, (int)SPICE_ERR_TIMEOUT);
    cluster_sync();   // the pair's MMAs, copies and signals are over in both CTAs; SPLIT: everybody's sums are there
    if constexpr (SPLIT) {
        if (warp >= 4 && pair < n_tiles) {
            // every CTA of the cluster finishes some of the tokens, a warp a token at a time
            const int ctas = 2 * g.split;
            const bool ok = *abort_flag == 0;
            int group = 0;
            const Tile t = find_tile(sh, g, pair, group);
            for (int c = (int)cluster_rank() + (warp - 4) * ctas; c < t.rows; c += PR_EPI_WARPS * ctas)
                finish_token<SWIGLU>(g, smem_u32(ring) + (c & 127) * (ST_RED_PITCH * 4), g.split, 2, c >> 7, (size_t)(t.t0 + c), t.nt, ok, lane);
        }
        cluster_sync();   // nobody leaves while a peer reads its sums
    }
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512));
}

// ------------------------------------------------------------------------------------------------ host side
std::atomic<uint32_t> wait_limit{WAIT_LIMIT};   // (SPICE_OPT_E4M3_WAIT_LIMIT)

template <typename F>
void for_each_stream_kernel(F f) {
    auto of = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        f((const void *)gemm_e4m3_stream_kernel<NT, false, false>, stream_smem<NT>());
        f((const void *)gemm_e4m3_stream_kernel<NT, true, false>, stream_smem<NT>());
        f((const void *)gemm_e4m3_stream_kernel<NT, false, true>, stream_smem<NT>());
        f((const void *)gemm_e4m3_stream_kernel<NT, true, true>, stream_smem<NT>());
    };
    of(std::integral_constant<int, 1>{});
    of(std::integral_constant<int, 2>{});
    of(std::integral_constant<int, 4>{});
}

// What a device is asked once: dynamic shared memory limits are raised, and how many clusters of c CTAs run at the same time when
// an SM holds one CTA.
struct DeviceFacts {
    std::atomic<bool> ready;
    int clusters[ST_MAX_SPLIT + 1];
};
const DeviceFacts *device_facts(int dev, int sms) {
    static DeviceFacts facts[64];
    static std::mutex mutex;
    DeviceFacts &f = facts[dev];
    if (f.ready.load(std::memory_order_acquire)) return &f;
    std::lock_guard<std::mutex> lock(mutex);
    if (f.ready.load(std::memory_order_relaxed)) return &f;
    bool ok = true;
    auto raise = [&](const void *kernel, size_t bytes) {
        ok = ok && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
    };
    for_each_stream_kernel(raise);
    raise((const void *)gemm_e4m3_pair_kernel<false, false>, PR_SMEM_BYTES);
    raise((const void *)gemm_e4m3_pair_kernel<true, false>, PR_SMEM_BYTES);
    raise((const void *)gemm_e4m3_pair_kernel<false, true>, PR_SMEM_BYTES);
    raise((const void *)gemm_e4m3_pair_kernel<true, true>, PR_SMEM_BYTES);
    for (int c = 2; ok && c <= ST_MAX_SPLIT; c *= 2) {   // (the larger of the two kernels)
        cudaLaunchConfig_t lc{};
        lc.gridDim = dim3((unsigned)(c * sms), 1, 1);
        lc.blockDim = dim3(PR_THREADS, 1, 1);
        lc.dynamicSmemBytes = PR_SMEM_BYTES;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)c;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        lc.attrs = at;
        lc.numAttrs = 1;
        ok = cudaOccupancyMaxActiveClusters(&f.clusters[c], gemm_e4m3_pair_kernel<false, true>, &lc) == cudaSuccess;
    }
    if (!ok) return nullptr;
    f.ready.store(true, std::memory_order_release);
    return &f;
}

template <int NT, bool SWIGLU>
bool launch_stream(GemmE4m3Args g, const CUtensorMap &map_w, const uint8_t *x, int64_t most, const DeviceFacts *facts, int sms, cudaStream_t st) {
    CUtensorMap map_x;
    if (!tc_encode_map2_bytes(&map_x, x, (uint64_t)g.T, (uint64_t)g.k, StreamShape<NT>::TOKENS)) return false;
    // a cluster takes one item, so all of them have to run at once
    g.split = 1;
    for (int c = 2; c <= ST_MAX_SPLIT; c *= 2)
        if (most <= facts->clusters[c] && g.kb >= 2 * c) g.split = c;
    if (g.split > 1)
        return launch_early(gemm_e4m3_stream_kernel<NT, SWIGLU, true>, dim3((unsigned)(most * g.split)), ST_THREADS, stream_smem<NT>(), st, g.split, map_w, map_x, g);
    return launch_early(gemm_e4m3_stream_kernel<NT, SWIGLU, false>, dim3((unsigned)std::min<int64_t>(sms, most)), ST_THREADS, stream_smem<NT>(), st, 1, map_w,
                        map_x, g);
}

template <bool SWIGLU>
spice_status launch_gemm_e4m3(GemmE4m3Args g, const uint8_t *x, const uint8_t *w, cudaStream_t st) {
    int dev = 0;
    const int sms = current_device_sms(&dev);
    if (sms <= 0) return SPICE_ERR_CUDA;
    const DeviceFacts *facts = device_facts(dev, sms);
    if (!facts) return SPICE_ERR_CUDA;
    const int w_rows = SWIGLU ? 2 * g.n : g.n;
    const int used = std::min(g.G, g.T);   // groups that can have rows
    const int rows = (g.T + used - 1) / used;
    if constexpr (!SWIGLU) {
        // A few tokens and few weights that can be touched: no ring.  Without / with it, us, one token: 512 x 1024 1.8/4.2,
        // 2048 x 2048 3.9/5.1, 8192 x 2048 5.8/7.3, 16384 x 2048 9.6/10.1 (in turns of two blocks also 2048 x 4096 6.8/6.4, 2048 x 8192
        // 10.3/8.0);  2048 x 1408 of 64 groups, 1 / 2 / 8 rows: 4.6/6.5, 5.2/7.7, 9.9/10.9;  4096 x 2048 of 8, 8 rows (64 MiB): 17.5/15.3.
        // (SwiGLU needs clusters for its blocks of 128 columns all the same: no gain.)
        if (g.T <= FEW_TOKENS && g.kb <= FEW_WARPS * FEW_BLOCKS && (int64_t)used * g.n * g.k <= (32 << 20)) {
            const dim3 grid((unsigned)((g.n + 15) / 16), (unsigned)used);
            return launch_early(gemm_e4m3_few_kernel, grid, FEW_WARPS * 32, 0, st, 1, x, w, g) ? SPICE_OK : SPICE_ERR_CUDA;
        }
    }
    // Few rows: streamed weights, at the rate of HBM as long as the warp-wide products (400 per cycle and SM) keep up.  Streamed / by
    // pairs of CTAs, us, dense 2048 x 2816, 3584 x 20480, SwiGLU 2816 x 2048:  16 tokens 6.8/10.0, 18.6/26.7, 8.0/11.6;  32 tokens
    // 9.4/10.6, 28.6/27.5, 11.0/12.0;  64 tokens (when it took them) 14.7/12.0, 56/29.5, -/13.3.  64 groups of 2048 x 1408, SwiGLU
    // 1408 x 2048:  96 rows 33.0/49, 59.6/94;  400 rows 37.8/50, 76.6/103;  768 rows 57/51, 116/103.
    if (g.G == 1 ? g.T <= 32 : rows <= 8) {
        CUtensorMap map_w;
        if (!tc_encode_map2_bytes(&map_w, w, (uint64_t)g.G * w_rows, (uint64_t)g.k, 128)) return SPICE_ERR_CUDA;
        g.n_tiles = SWIGLU ? g.n / 128 : (g.n + 255) / 256;
        auto most = [&](int tokens) {   // items there can be
            return g.G == 1 ? (int64_t)((g.T + tokens - 1) / tokens) * g.n_tiles : ((int64_t)g.T / tokens + used) * g.n_tiles;
        };
        if (most(8) > 0x3fffffff || (most(8) / sms + 1) * g.kb > 0x7fffffff) return SPICE_ERR_UNSUPPORTED_SHAPE;
        const int wide = g.G == 1 ? g.T : 2 * rows;   // (groups have unequal shares; a large one takes several items)
        const bool ok = wide <= 8 ? launch_stream<1, SWIGLU>(g, map_w, x, most(8), facts, sms, st)
                        : wide <= 16 ? launch_stream<2, SWIGLU>(g, map_w, x, most(16), facts, sms, st)
                                     : launch_stream<4, SWIGLU>(g, map_w, x, most(32), facts, sms, st);
        return ok ? SPICE_OK : SPICE_ERR_CUDA;
    }
    g.n_tiles = SWIGLU ? g.n / 128 : (g.n + PR_TILE - 1) / PR_TILE;
    const int row_bytes = SWIGLU ? 1 : g.out == SPICE_OUT_BF16 ? 2 : 4;
    g.sectors = ((reinterpret_cast<uintptr_t>(g.y) | (uintptr_t)g.n * row_bytes) & 31u) == 0;
    const int64_t most = (g.G == 1 ? ((int64_t)g.T + PR_TILE - 1) / PR_TILE : (int64_t)g.T / PR_TILE + used) * g.n_tiles;   // tiles there can be
    if (most > 0x3fffffff || (most / (sms / 2) + 1) * g.kb > 0x7fffffff) return SPICE_ERR_UNSUPPORTED_SHAPE;
    CUtensorMap map_w, map_x128, map_x16, map_y;
    if (!tc_encode_map2_bytes(&map_w, w, (uint64_t)g.G * w_rows, (uint64_t)g.k, 128) ||
        !tc_encode_map2_bytes(&map_x128, x, (uint64_t)g.T, (uint64_t)g.k, 128) ||
        !tc_encode_map2_bytes(&map_x16, x, (uint64_t)g.T, (uint64_t)g.k, 16) ||
        !tc_encode_map2_bytes(&map_y, g.y, (uint64_t)g.T, (uint64_t)g.n * row_bytes, 32))
        return SPICE_ERR_CUDA;
    // Fewer tiles than pairs: two or four pairs share a tile's reduction, as long as all the clusters run at once and the reduction is
    // long: 470 ns a block against a start of 4.5 us, or 6.8 with the cluster and 26 ns for a token's sums.  With one / two / four pairs
    // to a tile, us: 77 x 3584 x 20480 81 / 48 / 30, 256 tokens 76 / 57 / 37;  2048 x 2816 with 33 tokens 14.2 / 12.4 / 10.6, with 77
    // 15.4 / 13.5 / 12.5, with 256 15.4 / 17.4 / 16.6;  512 x 1024 with 77 8.5 / 9.6 / 9.4;  400 x 2048 x 8192 33.8 / 29.2.
    int share = 1;
    int64_t best = 4500 + 470 * (int64_t)g.kb;
    for (int s = 2; s <= 4 && g.G == 1; s *= 2) {
        const int64_t ns = 6800 + 26 * std::min(g.T, PR_TILE) + 470 * (int64_t)((g.kb + s - 1) / s);
        if (most <= facts->clusters[2 * s] && ns < best) {
            best = ns;
            share = s;
        }
    }
    bool ok;
    if (share > 1) {
        g.split = share;
        ok = launch_early(gemm_e4m3_pair_kernel<SWIGLU, true>, dim3((unsigned)(2 * share * most)), PR_THREADS, PR_SMEM_BYTES, st, 2 * share, map_w, map_x128,
                          map_x16, map_y, g);
    } else {
        const int pairs = (int)std::min<int64_t>(sms / 2, most);
        g.most_tiles = (uint32_t)std::min<int64_t>(g.most_tiles, (int64_t)(0x7fffffff / g.kb) * pairs);   // (a pair counts its blocks in 32 bits)
        ok = launch_early(gemm_e4m3_pair_kernel<SWIGLU, false>, dim3(2 * (unsigned)pairs), PR_THREADS, PR_SMEM_BYTES, st, 2, map_w, map_x128, map_x16, map_y, g);
    }
    return ok ? SPICE_OK : SPICE_ERR_CUDA;
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
    g.most_tiles = 1u << 30;
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
