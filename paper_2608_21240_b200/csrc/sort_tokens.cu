// Tokens sorted by expert and brought back with their weights, and the gradient of that.
//
//   entry i = t K + k of idx is kept iff 0 <= idx_i < N;   pos_i = number of kept j with (idx_j, j) < (idx_i, i);   entry[pos_i] = i
//   rows[pos_i] = x[t]                                            (the gather; its gradient is the sum below with weights of 1)
//   y[t] = sum_k gate[t,k] rows[pos[t,k]]
//   d_rows[pos[t,k]] = gate[t,k] dy[t],   d_gate[t,k] = <dy[t], rows[pos[t,k]]>
//
// The order is that of a stable sort, found by counting, without atomics on memory: the same input gives the same order.  What
// moves rows is bound by HBM; each row is read once and written once.
#include <algorithm>

#include "entry.cuh"
#include "spice_internal.cuh"
#include "tc_device.cuh"

namespace spice {

namespace {

struct SortArgs {
    const int32_t *idx;   // [T, K]
    int32_t *offset;      // [N + 1]
    int32_t *pos;         // [T, K]
    int32_t *entry;       // [T K]
    int32_t T, K, N, n;   // n = T K
    // the gather (rows: null without it)
    const uint4 *x;
    uint4 *rows;
    int32_t vecs;         // 16-byte pieces of a row
    const float *xs;      // scales that go with the rows, or null
    float *rs;
    int32_t ns;
};

__device__ __forceinline__ uint4 load16(const uint4 *p) {   // (not as constant: the kernel may be set up early)
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 load16_once(const uint4 *p) {   // (nobody reads it again)
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int32_t load4(const int32_t *p) {
    int32_t v;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load4(const float *p) {
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ int warp_sum(int v) { return __reduce_add_sync(0xffffffffu, v); }

// One token's row to its K places; pos: the places, in shared memory.
__device__ __forceinline__ void gather_row(const SortArgs &a, int t, const int32_t *pos) {
    for (int v = threadIdx.x; v < a.vecs; v += blockDim.x) {
        const uint4 x = load16(a.x + (size_t)t * a.vecs + v);
        for (int k = 0; k < a.K; ++k)
            if (pos[k] >= 0) a.rows[(size_t)pos[k] * a.vecs + v] = x;
    }
    if (!a.xs) return;
    for (uint32_t v = threadIdx.x; v < (uint32_t)a.ns; v += blockDim.x) {   // (up to 2^31 - 1 scales: the step behind them has to fit)
        const float x = load4(a.xs + (size_t)t * a.ns + v);
        for (int k = 0; k < a.K; ++k)
            if (pos[k] >= 0) a.rs[(size_t)pos[k] * a.ns + v] = x;
    }
}

// ------------------------------------------------------------------------------------------------ few entries
// A block per token: it counts the places of its own K entries among all of them (a warp per entry), and moves its row.  The
// last block counts the experts' entries beside its own.
constexpr int SMALL_N = 2048, SMALL_THREADS = 256;

__global__ void __launch_bounds__(SMALL_THREADS) sort_small_kernel(const SortArgs a) {
    __shared__ int32_t e[SMALL_N], place[32], hist[1024], part[SMALL_THREADS / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool counts = blockIdx.x == gridDim.x - 1;
    grid_dependency();
    if (counts)
        for (int i = threadIdx.x; i < a.N; i += SMALL_THREADS) hist[i] = 0;
    for (int i = threadIdx.x; i < a.n; i += SMALL_THREADS) {
        const int v = load4(a.idx + i);
        e[i] = v >= 0 && v < a.N ? v : INT32_MAX;   // dropped: behind everything
    }
    __syncthreads();
    const int t = blockIdx.x;
    for (int k = warp; k < a.K; k += SMALL_THREADS / 32) {
        const int i = t * a.K + k, own = e[i];
        int before = 0;
        for (int j = lane; j < a.n; j += 32) before += e[j] < own || (e[j] == own && j < i);
        before = warp_sum(before);
        if (lane == 0) {
            const int p = own != INT32_MAX ? before : -1;
            place[k] = p;
            a.pos[i] = p;
            if (p >= 0) a.entry[p] = i;
        }
    }
    __syncthreads();
    if (a.rows) gather_row(a, t, place);
    if (!counts) return;
    for (int i = threadIdx.x; i < a.n; i += SMALL_THREADS)
        if (e[i] != INT32_MAX) atomicAdd(&hist[e[i]], 1);
    __syncthreads();
    // a thread sums 4 experts; exclusive prefix sums over the threads
    int own[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = threadIdx.x * 4 + j;
        own[j] = i < a.N ? hist[i] : 0;
        sum += own[j];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) part[warp] = incl;
    __syncthreads();
    int base = incl - sum, kept = 0;
    for (int w = 0; w < SMALL_THREADS / 32; ++w) {
        if (w < warp) base += part[w];
        kept += part[w];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = threadIdx.x * 4 + j;
        if (i < a.N) a.offset[i] = base;
        base += own[j];
    }
    if (threadIdx.x == 0) a.offset[a.N] = kept;
    for (int i = kept + threadIdx.x; i < a.n; i += SMALL_THREADS) a.entry[i] = -1;
}

// ------------------------------------------------------------------------------------------------ many entries
// A cluster counts: each of its warps owns a run of consecutive entries and a row of counters in shared memory; a first pass
// counts, prefix sums over experts, blocks and warps turn the counters into places, a second pass hands the places out.  24576 entries
// of 64 experts 7.9 us; the other SMs wait, so the time grows with the entries: 65536 14.7, 262144 59.7 us.
constexpr int SORT_CTAS = 8, SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32, SORT_KEPT = 8, SORT_EXPERTS = 1024;
constexpr size_t sort_smem(int experts) { return (size_t)(SORT_WARPS * (experts | 1) + experts) * 4; }

__global__ void __launch_bounds__(SORT_THREADS, 1) sort_cluster_kernel(const SortArgs a) {
    extern __shared__ int32_t smem[];
    const int pitch = a.N | 1;                     // (odd: a column of counters falls into different banks)
    int32_t *mine = smem;                          // [warps][pitch] counters
    int32_t *total = smem + SORT_WARPS * pitch;    // [N] of this block
    __shared__ int32_t part[SORT_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = blockIdx.x;
    int32_t *own = mine + warp * pitch;
    for (int i = lane; i < a.N; i += 32) own[i] = 0;
    grid_dependency();
    const int share = (((a.n + SORT_CTAS * SORT_WARPS - 1) / (SORT_CTAS * SORT_WARPS)) + 31) & ~31;
    const int64_t from = (int64_t)(cta * SORT_WARPS + warp) * share;
    const int first = (int)min(from, (int64_t)a.n), last = (int)min(from + share, (int64_t)a.n);
    auto expert = [&](int i) {
        const int v = i < last ? load4(a.idx + i) : -1;
        return v >= 0 && v < a.N ? v : -1;
    };
    // the first entries of a warp stay in registers for the second pass
    int e[SORT_KEPT];
#pragma unroll
    for (int u = 0; u < SORT_KEPT; ++u) e[u] = expert(first + u * 32 + lane);
    __syncwarp();
    uint32_t kept_same[SORT_KEPT];
    auto count = [&](int v) {
        const uint32_t same = __match_any_sync(0xffffffffu, v);
        if (v >= 0 && (same & ((1u << lane) - 1)) == 0) own[v] += __popc(same);
        __syncwarp();
        return same;
    };
#pragma unroll
    for (int u = 0; u < SORT_KEPT; ++u)
        if (first + u * 32 < last) kept_same[u] = count(e[u]);
    for (int i = first + SORT_KEPT * 32; i < last; i += 32) count(expert(i + lane));
    __syncthreads();
    // counters of an expert: what the warps before have
    for (int x = warp; x < a.N; x += SORT_WARPS) {
        const int c = mine[lane * pitch + x];
        int incl = c;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        mine[lane * pitch + x] = incl - c;
        if (lane == 31) total[x] = incl;
    }
    tcdev::cluster_sync();
    int before = 0, all = 0;                       // entries of this thread's expert in earlier blocks, and in all
    if (threadIdx.x < a.N) {
        const uint32_t at = tcdev::smem_u32(total + threadIdx.x);
#pragma unroll
        for (int r = 0; r < SORT_CTAS; ++r) {
            int c;
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(c) : "r"(tcdev::map_to_cta(at, (uint32_t)r)));
            before += r < cta ? c : 0;
            all += c;
        }
    }
    int incl = all;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) part[warp] = incl;
    tcdev::cluster_sync();                         // (also: nobody's totals are needed any more)
    const int sums = part[lane];
    const int n_kept = warp_sum(sums), base = incl - all + warp_sum(lane < warp ? sums : 0);
    if (threadIdx.x < a.N) {
        if (cta == 0) a.offset[threadIdx.x] = base;
        total[threadIdx.x] = base + before;
    }
    if (cta == 0 && threadIdx.x == 0) a.offset[a.N] = n_kept;
    __syncthreads();
    auto place = [&](int i, int v, uint32_t same) {
        const uint32_t below = same & ((1u << lane) - 1);
        const int c = v >= 0 ? own[v] : 0;
        __syncwarp();
        if (v >= 0 && below == 0) own[v] = c + __popc(same);
        __syncwarp();
        if (i < last) {
            const int p = v >= 0 ? total[v] + c + __popc(below) : -1;
            a.pos[i] = p;
            if (p >= 0) a.entry[p] = i;
        }
    };
#pragma unroll
    for (int u = 0; u < SORT_KEPT; ++u)
        if (first + u * 32 < last) place(first + u * 32 + lane, e[u], kept_same[u]);
    for (int i = first + SORT_KEPT * 32; i < last; i += 32) {
        const int v = expert(i + lane);
        place(i + lane, v, __match_any_sync(0xffffffffu, v));
    }
    for (int i = n_kept + cta * SORT_THREADS + threadIdx.x; i < a.n; i += SORT_CTAS * SORT_THREADS) a.entry[i] = -1;
}

// A thread has one 16-byte piece (or scale) of a token.
__global__ void __launch_bounds__(256) gather_kernel(const SortArgs a) {
    grid_dependency();
    const int per = a.vecs + a.ns;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.T * per) return;
    const int t = (int)(i / per), v = (int)(i - (int64_t)t * per);
    const int32_t *pos = a.pos + (size_t)t * a.K;
    constexpr int U = 8;
    if (v < a.vecs) {
        const uint4 x = load16(a.x + (size_t)t * a.vecs + v);
        for (int k0 = 0; k0 < a.K; k0 += U) {
            int p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) p[u] = k0 + u < a.K ? load4(pos + k0 + u) : -1;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p[u] >= 0) a.rows[(size_t)p[u] * a.vecs + v] = x;
        }
    } else {
        const float x = load4(a.xs + (size_t)t * a.ns + v - a.vecs);
        for (int k = 0; k < a.K; ++k) {
            const int p = load4(pos + k);
            if (p >= 0) a.rs[(size_t)p * a.ns + v - a.vecs] = x;
        }
    }
}

// ------------------------------------------------------------------------------------------------ back
struct CombineRowsArgs {
    const void *rows;     // [n_rows, d]
    const int32_t *pos;   // [T, K]
    const float *gate;    // [T, K] or null
    void *y;              // [T, d]
    int32_t K, d, n_rows, out;
};

// eight consecutive values as fp32
template <bool F32>
struct Eight {
    uint4 v[F32 ? 2 : 1];
    __device__ __forceinline__ void load_once(const void *p, size_t at) {
        const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const char *>(p) + at * (F32 ? 4 : 2));
        v[0] = load16_once(q);
        if constexpr (F32) v[1] = load16_once(q + 1);
    }
    __device__ __forceinline__ void load(const void *p, size_t at) {
        const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const char *>(p) + at * (F32 ? 4 : 2));
        v[0] = load16(q);
        if constexpr (F32) v[1] = load16(q + 1);
    }
    __device__ __forceinline__ float operator[](int j) const {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(v);
        if constexpr (F32) return __uint_as_float(w[j]);
        else return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
    }
};
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&b);
}
template <bool F32>
__device__ __forceinline__ void store8(void *p, size_t at, const float (&f)[8]) {
    uint4 *q = reinterpret_cast<uint4 *>(static_cast<char *>(p) + at * (F32 ? 4 : 2));
    if constexpr (F32) {
        *reinterpret_cast<float4 *>(q) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4 *>(q + 1) = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        *q = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
    }
}

// A thread sums eight columns of a token; the rows of U entries are on their way at once.  Many tokens: two and as many blocks as fit
// (4096 x 6 x 2048: 19.7 us, 0.92 of the measured copy rate; six and five blocks 20.4; with the rows kept in L2 22 to 25).  Few: the
// shortest chain (17 x 8 x 3584: 2.0 us, with two at a time 2.6).
template <bool F32, int U>
__global__ void __launch_bounds__(256, U == 2 ? (F32 ? 5 : 8) : 1) combine_rows_kernel(const CombineRowsArgs a) {
    grid_dependency();
    const int t = blockIdx.x, col = (blockIdx.y * blockDim.x + threadIdx.x) * 8;
    if (col >= a.d) return;
    const int32_t *pos = a.pos + (size_t)t * a.K;
    const float *gate = a.gate ? a.gate + (size_t)t * a.K : nullptr;
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    for (int k0 = 0; k0 < a.K; k0 += U) {
        Eight<F32> r[U];
        float g[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = k0 + u < a.K ? load4(pos + k0 + u) : -1;
            in[u] = p >= 0 && p < a.n_rows;
            g[u] = in[u] && gate ? load4(gate + k0 + u) : 1.0f;
            if (in[u]) r[u].load_once(a.rows, (size_t)p * a.d + col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (in[u]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = fmaf(g[u], r[u][j], f[j]);
            }
    }
    const size_t at = (size_t)t * a.d + col;
    if (a.out == SPICE_OUT_BF16) {
        store8<false>(a.y, at, f);
    } else {
        if (a.out == SPICE_OUT_F32_ADD) {
            Eight<true> o;
            o.load(a.y, at);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] += o[j];
        }
        store8<true>(a.y, at, f);
    }
}

struct CombineGradArgs {
    const void *dy;       // [T, d]
    const void *rows;     // [n_rows, d]; null: the gates' gradient is not wanted
    const int32_t *pos;   // [T, K]
    const float *gate;    // [T, K] or null
    void *d_rows;         // [n_rows, d] or null
    float *d_gate;        // [T, K] or null
    int32_t n, K, d, n_rows;
};

// A block per entry, for few of them: its row of the gradient, and the product of dy with its row.
template <bool DY32, bool ROW32>
__global__ void __launch_bounds__(256) grad_entry_kernel(const CombineGradArgs a) {
    __shared__ float part[8];
    grid_dependency();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = blockIdx.x;
    const int p = load4(a.pos + i);
    float sum = 0.0f;
    if (p >= 0 && p < a.n_rows) {
        const float g = a.gate ? load4(a.gate + i) : 1.0f;
        const size_t from = (size_t)(i / a.K) * a.d, to = (size_t)p * a.d;
#pragma unroll 4
        for (int col = threadIdx.x * 8; col < a.d; col += 256 * 8) {
            Eight<DY32> dy;
            Eight<ROW32> r;
            dy.load(a.dy, from + col);
            if (a.d_gate) r.load(a.rows, to + col);
            if (a.d_rows) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = g * dy[j];
                store8<ROW32>(a.d_rows, to + col, f);
            }
            if (a.d_gate) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(dy[j], r[j], sum);
            }
        }
    }
    if (!a.d_gate) return;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.0f;
        for (int w = 0; w < 8; ++w) s += part[w];
        a.d_gate[i] = s;
    }
}

// A block per token, for many: dy is read once for all of the token's entries, three of which are on their way at once, with as many
// blocks as fit (4096 x 6 x 2048: 35.7 us, 0.95 of the measured copy rate; four at a time and five blocks 43.  fp32 67.8 us, at the copy
// rate; rows in fp32 and dy in bf16 65.7, 0.99; rows in bf16 and dy in fp32 43.9, 0.83).
template <bool DY32, bool ROW32>
__global__ void __launch_bounds__(256, ROW32 || DY32 ? 4 : 8) grad_token_kernel(const CombineGradArgs a) {
    __shared__ float part[8][32];
    grid_dependency();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.x;
    const int32_t *pos = a.pos + (size_t)t * a.K;
    const float *gate = a.gate ? a.gate + (size_t)t * a.K : nullptr;
    for (int c0 = 0; c0 < a.d; c0 += blockDim.x * 8) {
        const int col = c0 + threadIdx.x * 8;
        const bool in = col < a.d;
        Eight<DY32> dy;
        if (in) dy.load(a.dy, (size_t)t * a.d + col);
        constexpr int U = ROW32 ? 2 : 3;
        for (int k0 = 0; k0 < a.K; k0 += U) {
            Eight<ROW32> r[U];
            int p[U];
            float g[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                p[u] = k0 + u < a.K ? load4(pos + k0 + u) : -1;
                p[u] = p[u] < a.n_rows ? p[u] : -1;
                g[u] = gate && k0 + u < a.K ? load4(gate + k0 + u) : 1.0f;
                if (in && p[u] >= 0 && a.d_gate) r[u].load(a.rows, (size_t)p[u] * a.d + col);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (in && p[u] >= 0 && a.d_rows) {
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = g[u] * dy[j];
                    store8<ROW32>(a.d_rows, (size_t)p[u] * a.d + col, f);
                }
                if (!a.d_gate || k0 + u >= a.K) continue;
                float sum = 0.0f;
                if (in && p[u] >= 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fmaf(dy[j], r[u][j], sum);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane == 0) part[warp][k0 + u] = c0 ? part[warp][k0 + u] + sum : sum;
            }
        }
    }
    if (!a.d_gate) return;
    __syncthreads();
    if (threadIdx.x < a.K) {
        float s = 0.0f;
        for (int w = 0; w < (int)blockDim.x / 32; ++w) s += part[w][threadIdx.x];
        a.d_gate[(size_t)t * a.K + threadIdx.x] = s;
    }
}

bool misaligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
constexpr int64_t MAX_ENTRIES = 1 << 28;

// Raises the cluster kernel's limit on the current device to what the most experts take.  The limit belongs to the kernel, not to a
// call: all threads set the same value, so that none lowers it between another's setting and launch.
bool raise_sort_smem() {
    static std::atomic<bool> raised[64];
    int dev = 0;
    if (current_device_sms(&dev) <= 0) return false;
    if (raised[dev].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(sort_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sort_smem(SORT_EXPERTS)) != cudaSuccess) return false;
    raised[dev].store(true, std::memory_order_release);
    return true;
}

}  // namespace

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_sort_tokens(const int32_t *idx, int32_t T, int32_t top_k, int32_t n_experts, int32_t *offset,
                                          int32_t *pos, int32_t *entry, const void *x, int32_t row_bytes, void *rows,
                                          const float *x_scale, int32_t scale_cols, float *rows_scale, void *stream) {
    Range range_("spice_sort_tokens");
    if (T < 0 || top_k < 1 || n_experts < 1 || !offset || misaligned4(offset)) return SPICE_ERR_INVALID_ARG;
    if (n_experts > SORT_EXPERTS || top_k > 32 || (int64_t)T * top_k > MAX_ENTRIES) return SPICE_ERR_UNSUPPORTED_SHAPE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) return SPICE_OK;
    if (!x != !rows || (!x && (x_scale || rows_scale)) || !x_scale != !rows_scale || (x && (row_bytes < 16 || row_bytes % 16)) ||
        (x_scale && scale_cols < 1))
        return SPICE_ERR_INVALID_ARG;
    if (!idx || !pos || !entry || misaligned4(idx) || misaligned4(pos) || misaligned4(entry) || !aligned16(x) || !aligned16(rows) ||
        misaligned4(x_scale) || misaligned4(rows_scale))
        return SPICE_ERR_INVALID_ARG;
    const SortArgs a{idx, offset, pos, entry, T, top_k, n_experts, T * top_k, static_cast<const uint4 *>(x), static_cast<uint4 *>(rows),
                     x ? row_bytes / 16 : 0, x_scale, rows_scale, x_scale ? scale_cols : 0};
    if (a.n <= SMALL_N) return launch_early(sort_small_kernel, dim3((unsigned)T), SMALL_THREADS, 0, st, 1, a) ? SPICE_OK : SPICE_ERR_CUDA;
    const int64_t gather_blocks = ((int64_t)T * ((int64_t)a.vecs + a.ns) + 255) / 256;   // (fewer than 2^31: a sum that does not fit an int is refused)
    if (gather_blocks > 0x7fffffffLL) return SPICE_ERR_UNSUPPORTED_SHAPE;
    const size_t smem = sort_smem(n_experts);
    if (smem > 48 * 1024 && !raise_sort_smem()) return SPICE_ERR_CUDA;
    if (!launch_early(sort_cluster_kernel, dim3(SORT_CTAS), SORT_THREADS, smem, st, SORT_CTAS, a)) return SPICE_ERR_CUDA;
    if (rows && !launch_early(gather_kernel, dim3((unsigned)gather_blocks), 256, 0, st, 1, a)) return SPICE_ERR_CUDA;
    return SPICE_OK;
}

extern "C" spice_status spice_combine_tokens(const void *rows, int32_t rows_type, int32_t n_rows, const int32_t *pos, const float *gate,
                                             int32_t T, int32_t top_k, int32_t d, int32_t out, void *y, void *stream) {
    Range range_("spice_combine_tokens");
    if (T < 0 || n_rows < 0 || top_k < 1 || d < 8 || d % 8 || (rows_type != SPICE_OUT_BF16 && rows_type != SPICE_OUT_F32) ||
        (out != SPICE_OUT_BF16 && out != SPICE_OUT_F32 && out != SPICE_OUT_F32_ADD))
        return SPICE_ERR_INVALID_ARG;
    if (top_k > 32 || d > (1 << 24) || (int64_t)T * top_k > MAX_ENTRIES) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    if ((!rows && n_rows > 0) || !pos || !y || !aligned16(rows) || !aligned16(y) || misaligned4(pos) || misaligned4(gate))
        return SPICE_ERR_INVALID_ARG;
    const CombineRowsArgs a{rows, pos, gate, y, top_k, d, n_rows, out};
    const int vecs = d / 8, threads = std::min(256, (vecs + 31) & ~31);
    const dim3 grid((unsigned)T, (unsigned)((vecs + threads - 1) / threads));
    const int sms = current_device_sms();
    if (sms <= 0) return SPICE_ERR_CUDA;
    const bool many = (int64_t)grid.x * grid.y >= 4 * sms;
    auto *kernel = rows_type == SPICE_OUT_F32 ? (many ? combine_rows_kernel<true, 2> : combine_rows_kernel<true, 4>)
                                              : (many ? combine_rows_kernel<false, 2> : combine_rows_kernel<false, 8>);
    return launch_early(kernel, grid, threads, 0, static_cast<cudaStream_t>(stream), 1, a) ? SPICE_OK : SPICE_ERR_CUDA;
}

extern "C" spice_status spice_combine_tokens_grad(const void *dy, int32_t dy_type, const void *rows, int32_t rows_type, int32_t n_rows,
                                                  const int32_t *pos, const float *gate, int32_t T, int32_t top_k, int32_t d,
                                                  void *d_rows, float *d_gate, void *stream) {
    Range range_("spice_combine_tokens_grad");
    if (T < 0 || n_rows < 0 || top_k < 1 || d < 8 || d % 8 || (dy_type != SPICE_OUT_BF16 && dy_type != SPICE_OUT_F32) ||
        (rows_type != SPICE_OUT_BF16 && rows_type != SPICE_OUT_F32))
        return SPICE_ERR_INVALID_ARG;
    if (top_k > 32 || d > (1 << 24) || (int64_t)T * top_k > MAX_ENTRIES) return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    if (!dy || !pos || (n_rows > 0 && ((!rows && d_gate) || (!d_rows && !d_gate))) || !aligned16(dy) || !aligned16(rows) || !aligned16(d_rows) || misaligned4(pos) ||
        misaligned4(gate) || misaligned4(d_gate))
        return SPICE_ERR_INVALID_ARG;
    const CombineGradArgs a{dy, rows, pos, gate, d_rows, d_gate, T * top_k, top_k, d, n_rows};
    if (!d_rows && !d_gate) return SPICE_OK;   // (no rows)
    const bool d32 = dy_type == SPICE_OUT_F32, r32 = rows_type == SPICE_OUT_F32;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.n < 2048) {
        auto *kernel = d32 ? (r32 ? grad_entry_kernel<true, true> : grad_entry_kernel<true, false>)
                           : (r32 ? grad_entry_kernel<false, true> : grad_entry_kernel<false, false>);
        return launch_early(kernel, dim3((unsigned)a.n), 256, 0, st, 1, a) ? SPICE_OK : SPICE_ERR_CUDA;
    }
    auto *kernel = d32 ? (r32 ? grad_token_kernel<true, true> : grad_token_kernel<true, false>)
                       : (r32 ? grad_token_kernel<false, true> : grad_token_kernel<false, false>);
    const int threads = std::min(256, (d / 8 + 31) & ~31);
    return launch_early(kernel, dim3((unsigned)T), threads, 0, st, 1, a) ? SPICE_OK : SPICE_ERR_CUDA;
}
