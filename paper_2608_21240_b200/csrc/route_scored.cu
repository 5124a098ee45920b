// Routing by scores: softmax or sigmoid scores of router logits, an optional bias that takes part in the selection only,
// optional groups of experts, top-k, weights that may be renormalised over the winners and scaled.
//
//   score_e = softmax(l)_e or sigmoid(l_e);   key_e = score_e + bias_e (without a bias: the order of l_e, which is theirs)
//   groups:   value = the largest key, or the sum of the two largest score_e + bias_e; the top_groups best groups stay
//   winners:  the top_k largest keys among the experts that stay, in order; equal keys towards the smaller index
//   gate_k  = scale * score_k, or scale * score_k / sum over the winners (0 when that sum is 0)
//
// An expert whose logit is NaN or -inf (or whose bias is) is unavailable: it ranks behind every other expert and has
// score 0, so a row that a mask leaves nothing still yields valid expert ids with gates of 0.
//
// Selection is a comparison of real numbers; fp32 scores decide it wherever two of them are further apart than their
// error bound.  Where two neighbours of the order are nearer than that, every expert that could be among the winners is
// evaluated by the same formulas in fp64, one per lane, and ranked (slow_row, a row at a time, where more than 32 could
// be); so are the groups where the last one that stays and the first that does not are that close.  Where the order is
// that of the logits nothing is rounded and the first answer stands.
//
// One warp per token.  Keys live in registers; a round of the selection is one warp-wide maximum of the keys and one minimum of
// the places that hold it (NaN marks a key that is out of the race: it is no maximum and equals nothing).  With groups, the keys
// pass through shared memory and only those of the groups that stay are read back.  Bytes are few (4 N per token, 1.4 us for
// 8192 x 256, which takes 12.9 us with a bias and groups): the time goes into the issue of some 1000 instructions per warp.
#include <cfloat>

#include "entry.cuh"
#include "spice_internal.cuh"

namespace spice {

namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int WARPS = 4;

struct RouteArgs {
    const float *logits;   // [T, N]
    const float *bias;     // [N] or null
    int32_t *idx;          // [T, K]
    float *gate;           // [T, K]
    int32_t T, N, K, n_groups, top_groups, norm_topk, sigmoid, pair;
    int32_t size;          // experts of a group
    int32_t lanes_log2;    // 2^lanes_log2 lanes share a group when the groups are weighed
    uint32_t size_magic;   // ceil(2^32 / (N / n_groups)): e / size as a high product (exact for e < 1024); 0 for size 1
    float scale;
};

// the largest of a warp's values, NaN only where all are
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float none() { return __uint_as_float(0x7fffffffu); }
__device__ __forceinline__ unsigned long long ordered64(double v) {
    const long long b = __double_as_longlong(v);
    return (unsigned long long)b ^ ((unsigned long long)(b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

__device__ __forceinline__ int group_of(const RouteArgs &a, int e) {
    return a.size_magic ? (int)__umulhi((uint32_t)e, a.size_magic) : e;
}

// best (key, lowest index) over the warp
__device__ __forceinline__ void warp_best64(unsigned long long &key, int &e) {
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long k2 = __shfl_xor_sync(FULL, key, o);
        const int e2 = __shfl_xor_sync(FULL, e, o);
        if (k2 > key || (k2 == key && e2 < e)) {
            key = k2;
            e = e2;
        }
    }
}

// the first of the lanes that share group g when the groups are weighed
__device__ __forceinline__ int first_lane(const RouteArgs &a, int g) { return (g << a.lanes_log2) & 31; }

// What the groups' values are made of, for the n_groups groups of `size` keys in shared memory: lane g gets group g's value,
// lane first_lane(g), in `terms`, the magnitudes of the keys that it is made of (a sum of two may be far smaller than they are).
template <typename F>
__device__ __forceinline__ F group_value(const RouteArgs &a, const F *keys, int size, int lane, F &terms) {
    // `width` lanes share a group: each looks at every width-th member, then they merge
    const int G = a.n_groups, width = 1 << a.lanes_log2;
    const int g = lane >> a.lanes_log2;
    F b0 = -(F)INFINITY, b1 = b0;   // the two largest
    if (g < G) {
        for (int j = lane & (width - 1); j < size; j += width) {
            const F x = keys[g * size + j];
            b1 = max(b1, min(b0, x));
            b0 = max(b0, x);
        }
    }
    for (int o = width >> 1; o > 0; o >>= 1) {
        const F o0 = __shfl_xor_sync(FULL, b0, o), o1 = __shfl_xor_sync(FULL, b1, o);
        b1 = max(max(b1, o1), min(b0, o0));
        b0 = max(b0, o0);
    }
    const bool both = a.pair && b1 > -(F)INFINITY;
    F value = both ? b0 + b1 : b0;
    if (both && value == -(F)INFINITY) value = -(F)FLT_MAX;   // two keys at the low end of fp32: not a group without an expert
    terms = both ? fabs(b0) + fabs(b1) : fabs(b0);
    return __shfl_sync(FULL, value, first_lane(a, lane));
}

// Rank of lane's key among those of lanes 0..n-1 (equal keys: the smaller `tag` first).
template <typename F>
__device__ __forceinline__ int rank_of(F key, int tag, int n) {
    int rank = 0;
    for (int j = 0; j < n; ++j) {
        const F k = __shfl_sync(FULL, key, j);
        const int t = __shfl_sync(FULL, tag, j);
        rank += k > key || (k == key && t < tag) ? 1 : 0;
    }
    return rank;
}

// fp64 scores of a row: softmax's largest logit and sum, then any expert's key
struct Score64 {
    double m, s;
    __device__ __noinline__ Score64(const RouteArgs &a, const float *l, int lane) : m(-(double)INFINITY), s(0.0) {
        if (a.sigmoid) return;
        for (int e = lane; e < a.N; e += 32)
            if (available(a, l, e)) m = fmax(m, (double)l[e]);
        for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(FULL, m, o));
        for (int e = lane; e < a.N; e += 32)
            if (available(a, l, e)) s += (double)l[e] == m ? 1.0 : exp((double)l[e] - m);
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
    }
    static __device__ __forceinline__ bool available(const RouteArgs &a, const float *l, int e) {
        return l[e] > -INFINITY && (!a.bias || a.bias[e] > -INFINITY);   // NaN compares false
    }
    __device__ __noinline__ double key(const RouteArgs &a, const float *l, int e) const {
        if (!available(a, l, e)) return -(double)INFINITY;
        const double v = l[e];
        const double sc = a.sigmoid ? 1.0 / (1.0 + exp(-v)) : (v == m ? 1.0 : exp(v - m)) / s;
        return sc + (a.bias ? (double)a.bias[e] : 0.0);
    }
};

// The groups that stay, in fp64.  keys: [N] doubles of this warp in shared memory.
__device__ __noinline__ uint32_t slow_groups(const RouteArgs &a, const float *l, double *keys, int size, int lane) {
    const Score64 sc(a, l, lane);
    __syncwarp();
    for (int e = lane; e < a.N; e += 32) keys[e] = sc.key(a, l, e);
    __syncwarp();
    double terms;
    const double v = group_value<double>(a, keys, size, lane, terms);
    const int rank = rank_of<double>(v, lane, a.n_groups);
    return __ballot_sync(FULL, lane < a.n_groups && rank < a.top_groups);
}

// The winners of one row in fp64 among the experts of the open groups, round by round: rows in which more than 32 experts
// could be among them (many equal keys).  Returns lane k's winner k.
__device__ __noinline__ int slow_row(const RouteArgs &a, const float *l, double *keys, uint32_t open, int lane) {
    const Score64 sc(a, l, lane);
    __syncwarp();
    for (int e = lane; e < a.N; e += 32) keys[e] = sc.key(a, l, e);
    int mine = 0;
    for (int i = 0; i < a.K; ++i) {
        __syncwarp();
        unsigned long long k = 0;
        int e = a.N;
        for (int j = lane; j < a.N; j += 32) {
            const double v = keys[j];
            if (v != v || !((open >> group_of(a, j)) & 1u)) continue;   // NaN: taken
            const unsigned long long kj = ordered64(v);
            if (kj > k) {
                k = kj;
                e = j;
            }
        }
        warp_best64(k, e);
        if (lane == i) mine = e;
        if (lane == 0) keys[e] = __longlong_as_double(0x7ff8000000000000ll);
    }
    __syncwarp();
    return mine;
}

// fast exponential and sigmoid: the keys' error bound covers them (the gates use the accurate functions)
__device__ __forceinline__ float fast_exp(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
    return y;
}
__device__ __forceinline__ float fast_sigmoid(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.0f + fast_exp(-x)));
    return y;
}

// V: experts per lane (e = lane + 32 i).  VS: keys per lane in the selection, those of the groups that stay
template <int V, int VS>
__global__ void __launch_bounds__(WARPS * 32) route_scored_kernel(const RouteArgs a) {
    extern __shared__ double sh_keys[];   // with groups or a bias: [WARPS][N] doubles, also the fp32 keys; then the open groups
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long t = (long long)blockIdx.x * WARPS + warp;
    grid_dependency();
    if (t >= a.T) return;   // warp-uniform; no block-wide barrier below
    const float *l = a.logits + (size_t)t * a.N;
    double *shd = sh_keys + (size_t)warp * a.N;
    float *shf = reinterpret_cast<float *>(shd);
    const int N = a.N, K = a.K;
    const bool grouped = a.n_groups > 1, by_score = a.bias != nullptr || a.pair;   // else everything goes by the logits

    float v[V], b[V];   // (b: only with a bias)
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        v[i] = e < N ? l[e] : -INFINITY;
        b[i] = a.bias && e < N ? a.bias[e] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (!(v[i] > -INFINITY) || !(b[i] > -INFINITY)) v[i] = -INFINITY;   // NaN too
    // ---- scores and keys
    float m = -INFINITY, inv = 1.0f;
    if (!a.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) m = fmaxf(m, v[i]);
        m = warp_max(m);
        if (by_score || !a.norm_topk) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[i] == m ? (m > -INFINITY ? 1.0f : 0.0f) : fast_exp(v[i] - m);
            s = warp_add(s);
            inv = s > 0.0f ? __fdividef(1.0f, s) : 0.0f;
        }
    }
    // Two keys nearer than tol (plus the rounding of score + bias) are not told apart.  A sigmoid score is off by at most
    // s (1 - s) (1.2 |x| + 2) 2^-23 from the exponential and 1.5 * 2^-23 s from sum and reciprocal: below 3.5e-7.  A
    // softmax score by (1.2 |x| + 2) 2^-23 e^x / sum, with |x| e^x < 0.37, and the V + 5 additions and the quotient: below
    // (13 + V) / 2 * 2^-23 of the largest score.
    const float tol = a.sigmoid ? 1e-6f : (13 + V) * 1.2e-7f * inv;
    float key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        float val = v[i];
        if (by_score && v[i] > -INFINITY)
            val = (a.sigmoid ? fast_sigmoid(v[i]) : (v[i] == m ? 1.0f : fast_exp(v[i] - m)) * inv) + b[i];
        if (grouped && e < N) shf[e] = val;
        key[i] = e < N ? (a.bias ? val : v[i]) : none();
    }
    // ---- groups: only the keys of those that stay are read back (in the order of the experts)
    float sel[VS];
    uint32_t open = FULL;
    int count = N;
    const int size = a.size;
    int32_t *list = reinterpret_cast<int32_t *>(sh_keys + (size_t)WARPS * N) + warp * 32;
    if (grouped) {
        __syncwarp();
        const int G = a.n_groups;
        float terms;
        const float mine = group_value<float>(a, shf, size, lane, terms);
        float left = lane < G ? mine : none();
        open = 0u;
        for (int i = 0; i < a.top_groups; ++i) {
            const float best_left = warp_max(left);
            const int best = __ffs(__ballot_sync(FULL, left == best_left)) - 1;
            open |= 1u << best;
            if (lane == best) left = none();
        }
        // A group's value is off by at most `off`: a score of each of its keys (tol / 2), the rounding of each key and that of
        // their sum (2^-24 of the keys' magnitudes each).  The choice stands where no group that does not stay can be worth as
        // much as one that does.
        bool call = false;   // warp-uniform
        if (by_score && a.top_groups < G) {
            const float off = fminf(tol + 2.4e-7f * __shfl_sync(FULL, terms, first_lane(a, lane)), 3e38f);
            const float out = warp_max(left + off), in = -warp_max((open >> lane) & 1u ? off - mine : none());
            call = out > -INFINITY && !(in > out);
        }
        if (call) open = slow_groups(a, l, shd, size, lane);
        if (call || (a.pair && !a.bias)) {
            // the winners' keys again: the doubles lay over them; or, without a bias, the logits in the place of the scores
            __syncwarp();
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane + 32 * i < N) shf[lane + 32 * i] = key[i];
        }
        if ((open >> lane) & 1u) list[__popc(open & ((1u << lane) - 1u))] = lane;
        __syncwarp();
        count = a.top_groups * size;
#pragma unroll
        for (int i = 0; i < VS; ++i) {
            const int c = lane + 32 * i;
            sel[i] = none();
            if (c < count) {
                const int og = group_of(a, c);
                sel[i] = shf[list[og] * size + c - og * size];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VS; ++i) sel[i] = i < V ? key[i < V ? i : 0] : none();
    }
    // ---- winners: lane k keeps the k-th, its place among the candidates and its key
    int win = 0;
    float won = none();
    auto round = [&](int k) {
        float best = sel[0];
#pragma unroll
        for (int i = 1; i < VS; ++i) best = fmaxf(best, sel[i]);
        const float top = warp_max(best);
        int at = 0x7fffffff;
#pragma unroll
        for (int i = VS - 1; i >= 0; --i)
            if (sel[i] == top) at = lane + 32 * i;
        at = __reduce_min_sync(FULL, at);   // equal keys: the smaller index
        if (lane == k) {
            win = at;
            won = top;
        }
#pragma unroll
        for (int i = 0; i < VS; ++i)
            if (at == lane + 32 * i) sel[i] = none();
        return top;
    };
    // whether a key is not told apart from the one before it in the order (NaN: there is none)
    auto near = [&](float x, float y) { return y > -INFINITY && x - y <= tol + 1.2e-7f * (fabsf(x) + fabsf(y)); };
    for (int k = 0; k < K; ++k) round(k);
    int have = K;
    bool close = false, many = false;
    if (a.bias) {
        // the first that is left is a possible winner too if the K-th is not told apart from it, and so on
        const float last = __shfl_sync(FULL, won, K - 1), before = __shfl_up_sync(FULL, won, 1);
        close = __any_sync(FULL, lane > 0 && lane < K && near(before, won));
        while (true) {
            if (have == 32) {   // no lane left: are there more?
                float best = sel[0];
#pragma unroll
                for (int i = 1; i < VS; ++i) best = fmaxf(best, sel[i]);
                many = near(last, warp_max(best));
                close |= many;
                break;
            }
            if (!near(last, round(have))) break;
            close = true;
            ++have;
        }
    }
    if (grouped && lane < have) {
        const int og = group_of(a, win);
        win = list[og] * size + win - og * size;
    }
    if (close) {   // warp-uniform
        if (many) {
            win = slow_row(a, l, shd, open, lane);
        } else {
            const Score64 sc(a, l, lane);
            const double k64 = lane < have ? sc.key(a, l, win) : 0.0;
            const int rank = rank_of<double>(k64, win, have);
            // lane `rank` takes this lane's expert
            int32_t *order = reinterpret_cast<int32_t *>(shf);
            __syncwarp();
            if (lane < have) order[rank] = win;
            __syncwarp();
            win = lane < K ? order[lane] : 0;
        }
    }
    // ---- gates
    float x = -INFINITY, g = 0.0f;
    if (lane < K) {
        x = l[win];
        if (!(x > -INFINITY) || (a.bias && !(a.bias[win] > -INFINITY))) x = -INFINITY;
    }
    const bool has = x > -INFINITY;
    if (a.norm_topk) {
        // relative to the winners' largest, so that a row of tiny scores keeps its ratios:
        // softmax: e^(x - M); sigmoid: e^(min(x,0) - M) / (1 + e^-|x|)
        const float y = a.sigmoid ? fminf(x, 0.0f) : x;
        const float M = warp_max(y);
        if (has) {
            g = y == M ? 1.0f : expf(y - M);
            if (a.sigmoid) g = __fdividef(g, 1.0f + expf(-fabsf(x)));
        }
        const float s = warp_add(g);
        g = s > 0.0f ? __fdividef(g, s) : 0.0f;
    } else if (has) {
        g = a.sigmoid ? __fdividef(1.0f, 1.0f + expf(-x)) : (x == m ? 1.0f : expf(x - m)) * inv;
    }
    if (lane < K) {
        a.idx[(size_t)t * K + lane] = win;
        a.gate[(size_t)t * K + lane] = a.scale * g;
    }
}

template <int V>
bool launch_route_scored(const RouteArgs &a, int vs, unsigned grid, size_t smem, cudaStream_t st) {
    auto *kernel = V >= 8 && vs <= V / 4 ? route_scored_kernel<V, (V >= 8 ? V / 4 : V)>
                   : V >= 4 && vs <= V / 2 ? route_scored_kernel<V, (V >= 4 ? V / 2 : V)> : route_scored_kernel<V, V>;
    return launch_early(kernel, dim3(grid), WARPS * 32, smem, st, 1, a);
}

}  // namespace

}  // namespace spice

using namespace spice;

extern "C" spice_status spice_route_scored(const float *logits, const float *bias, int32_t T, int32_t n_experts, int32_t top_k,
                                           int32_t score, int32_t n_groups, int32_t top_groups, int32_t group_score,
                                           int32_t norm_topk, float scale, int32_t *idx, float *gate, void *stream) {
    Range range_("spice_route_scored");
    if (T < 0 || (score != SPICE_SCORE_SOFTMAX && score != SPICE_SCORE_SIGMOID) ||
        (group_score != SPICE_GROUP_MAX && group_score != SPICE_GROUP_TOP2))
        return SPICE_ERR_INVALID_ARG;
    if (n_experts < 1 || n_experts > 1024 || top_k < 1 || top_k > 32 || n_groups < 1 || n_groups > 32 || n_experts % n_groups ||
        top_groups < 1 || top_groups > n_groups || top_k > top_groups * (n_experts / n_groups))
        return SPICE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return SPICE_OK;
    auto aligned4 = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; };
    if (!logits || !idx || !gate || !aligned4(logits) || !aligned4(bias) || !aligned4(idx) || !aligned4(gate))
        return SPICE_ERR_INVALID_ARG;
    const uint32_t size = (uint32_t)(n_experts / n_groups);
    const int pair = n_groups > 1 && group_score == SPICE_GROUP_TOP2;
    int lanes_log2 = 5;
    while (lanes_log2 > 0 && (n_groups << lanes_log2) > 32) --lanes_log2;
    const RouteArgs a{logits, bias, idx, gate, T, n_experts, top_k, n_groups, top_groups, norm_topk, score == SPICE_SCORE_SIGMOID, pair,
                      (int32_t)size, lanes_log2, size > 1 ? (uint32_t)((0x100000000ull + size - 1) / size) : 0u, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned grid = ((unsigned)T + WARPS - 1) / WARPS;
    const size_t smem = n_groups > 1 || bias ? (size_t)WARPS * (n_experts * sizeof(double) + 32 * sizeof(int32_t)) : 0;   // up to 33 KB
    const int v = (n_experts + 31) / 32, vs = (int)(top_groups * size + 31) / 32;
    const bool ok = v <= 2 ? launch_route_scored<2>(a, vs, grid, smem, st) : v <= 4 ? launch_route_scored<4>(a, vs, grid, smem, st)
                    : v <= 8 ? launch_route_scored<8>(a, vs, grid, smem, st) : v <= 16 ? launch_route_scored<16>(a, vs, grid, smem, st)
                    : launch_route_scored<32>(a, vs, grid, smem, st);
    return ok ? SPICE_OK : SPICE_ERR_CUDA;
}
