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
// error bound.  A row in which two neighbours of the order (or the last group that stays and the first that does not) are
// nearer than that is decided by the same formulas in fp64 (slow_row; about one row in a thousand at 256 experts).
// Where the order is that of the logits nothing is rounded and the first answer stands.
//
// One warp per token; keys live in registers as integers that order like the floats, a round of the selection is one
// warp-wide integer maximum for the key and one minimum for the index.  Bytes are few (4 N per token): the bound is the
// issue of the K + 1 rounds.
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
    int32_t T, N, K, n_groups, top_groups, norm_topk;
    uint32_t size_magic;   // ceil(2^32 / (N / n_groups)): e / size as a high product (exact for e < 1024); 0 for size 1
    float scale;
};

// integers in the order of the floats; 0 is below every float and marks what is out of the race
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
    return __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
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

// The selection of one row in fp64, for rows whose fp32 scores are too close to call.  key: [N] doubles of this warp in
// shared memory.  Returns the winners, lane k holding the k-th.
template <bool SIGMOID, bool PAIR>
__device__ __noinline__ int slow_row(const RouteArgs &a, const float *l, double *key, int lane) {
    const double ninf = -(double)INFINITY;
    double m = ninf, s = 0.0;
    if (!SIGMOID) {
        for (int e = lane; e < a.N; e += 32)
            if (l[e] > -INFINITY) m = fmax(m, (double)l[e]);
        for (int o = 16; o > 0; o >>= 1) m = fmax(m, __shfl_xor_sync(FULL, m, o));
        for (int e = lane; e < a.N; e += 32)
            if (l[e] > -INFINITY) s += (double)l[e] == m ? 1.0 : exp((double)l[e] - m);
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
    }
    for (int e = lane; e < a.N; e += 32) {
        const double v = l[e];
        const double sc = SIGMOID ? 1.0 / (1.0 + exp(-v)) : (v == m ? 1.0 : exp(v - m)) / s;
        const double k = sc + (a.bias ? (double)a.bias[e] : 0.0);
        key[e] = v > ninf && k > ninf ? k : ninf;
    }
    __syncwarp();
    uint32_t open = FULL;
    const int size = a.N / a.n_groups;
    if (a.n_groups > 1) {
        unsigned long long gk = 0;   // lane g: the value of group g
        if (lane < a.n_groups) {
            double b0 = ninf, b1 = ninf;
            for (int j = 0; j < size; ++j) {
                const double v = key[lane * size + j];
                if (v > b0) {
                    b1 = b0;
                    b0 = v;
                } else if (v > b1) {
                    b1 = v;
                }
            }
            gk = ordered64(PAIR && b1 > ninf ? b0 + b1 : b0);
        }
        open = 0;
        for (int i = 0; i < a.top_groups; ++i) {
            unsigned long long k = gk;
            int g = lane;
            warp_best64(k, g);
            open |= 1u << g;
            if (lane == g) gk = 0;
        }
    }
    if (!a.bias) {   // the winners' order is that of the logits (fp64 scores of large ones may coincide)
        __syncwarp();
        for (int e = lane; e < a.N; e += 32) key[e] = l[e] > -INFINITY ? (double)l[e] : ninf;
        __syncwarp();
    }
    int mine = 0;
    for (int i = 0; i < a.K; ++i) {
        unsigned long long k = 0;
        int e = a.N;
        for (int j = lane; j < a.N; j += 32) {
            if (a.n_groups > 1 && !((open >> group_of(a, j)) & 1u)) continue;
            const double v = key[j];
            if (v != v) continue;   // taken
            const unsigned long long kj = ordered64(v);
            if (kj > k) {
                k = kj;
                e = j;
            }
        }
        warp_best64(k, e);
        if (lane == i) mine = e;
        __syncwarp();
        if (lane == 0) key[e] = __longlong_as_double(0x7ff8000000000000ll);
        __syncwarp();
    }
    return mine;
}

// V: experts per lane (e = lane + 32 i)
template <int V, bool SIGMOID, bool PAIR>
__global__ void __launch_bounds__(WARPS * 32) route_scored_kernel(const RouteArgs a) {
    extern __shared__ double sh_keys[];   // [WARPS][N], also the fp32 values of a row's groups
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long t = (long long)blockIdx.x * WARPS + warp;
    if (t >= a.T) return;   // warp-uniform; no block-wide barrier below
    const float *l = a.logits + (size_t)t * a.N;
    double *shd = sh_keys + (size_t)warp * a.N;
    float *shf = reinterpret_cast<float *>(shd);
    const int N = a.N, K = a.K;

    float v[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        v[i] = e < N ? l[e] : -INFINITY;
        b[i] = a.bias && e < N ? a.bias[e] : 0.0f;
        if (!(v[i] > -INFINITY) || !(b[i] > -INFINITY)) v[i] = -INFINITY;   // NaN too
    }
    // ---- scores
    float m = -INFINITY, inv = 1.0f;
    const bool by_score = a.bias != nullptr || PAIR;   // else everything goes by the logits
    if (!SIGMOID) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, ordered(v[i]));
        m = unordered(__reduce_max_sync(FULL, top));
        if (by_score || !a.norm_topk) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) s += v[i] == m ? (m > -INFINITY ? 1.0f : 0.0f) : expf(v[i] - m);
            s = warp_add(s);
            inv = s > 0.0f ? 1.0f / s : 0.0f;
        }
    }
    uint32_t key[V];
    float tol = 0.0f;    // keys nearer than this (plus their own rounding) are not told apart
    if (by_score) {
        // expf within 2 ulp, its argument and the sums and quotients behind it: below (13 + V) half ulps of the score
        tol = SIGMOID ? 2e-6f : (13 + V) * 1.2e-7f * inv;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float sc = SIGMOID ? 1.0f / (1.0f + expf(-v[i])) : (v[i] == m ? 1.0f : expf(v[i] - m)) * inv;
            const float val = v[i] > -INFINITY ? sc + b[i] : -INFINITY;
            const int e = lane + 32 * i;
            key[i] = e < N ? ordered(a.bias ? val : v[i]) : 0u;
            if (PAIR && e < N) shf[e] = val;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = lane + 32 * i < N ? ordered(v[i]) : 0u;
    }
    bool close = false;
    // ---- groups
    if (a.n_groups > 1) {
        const int G = a.n_groups, size = N / G;
        if (!PAIR) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane + 32 * i < N) shf[lane + 32 * i] = unordered(key[i]);
        }
        __syncwarp();
        // `width` lanes share a group: each looks at every width-th member, then they merge
        const int width = G <= 1 ? 32 : 32 >> (32 - __clz(G - 1));
        const int g = lane / width;
        float b0 = -INFINITY, b1 = -INFINITY;
        if (g < G) {
            for (int j = lane & (width - 1); j < size; j += width) {
                const float x = shf[g * size + j];
                if (PAIR) b1 = fmaxf(b1, fminf(b0, x));
                b0 = fmaxf(b0, x);
            }
        }
        for (int o = width >> 1; o > 0; o >>= 1) {
            const float o0 = __shfl_xor_sync(FULL, b0, o);
            if (PAIR) {
                const float o1 = __shfl_xor_sync(FULL, b1, o);
                b1 = fmaxf(fmaxf(b1, o1), fminf(b0, o0));
            }
            b0 = fmaxf(b0, o0);
        }
        const float value = PAIR && b1 > -INFINITY ? b0 + b1 : b0;
        const float mine = __shfl_sync(FULL, value, (lane * width) & 31);   // lane g: group g
        uint32_t gk = lane < G ? ordered(mine) : 0u, open = 0, last = 0;
        for (int i = 0; i < a.top_groups; ++i) {
            last = __reduce_max_sync(FULL, gk);
            const int best = __ffs(__ballot_sync(FULL, gk == last)) - 1;
            open |= 1u << best;
            if (lane == best) gk = 0u;
        }
        if (by_score && a.top_groups < G) {
            const float in = unordered(last), out = unordered(__reduce_max_sync(FULL, gk));
            if (out > -INFINITY && in - out <= 2.0f * tol + 2.4e-7f * (fabsf(in) + fabsf(out))) close = true;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 32 * i;
            if (e < N && !((open >> group_of(a, e)) & 1u)) key[i] = 0u;
        }
    }
    // ---- winners: lane k keeps the k-th
    int win = 0;
    uint32_t before = 0;
    const bool check = a.bias != nullptr;
    const int rounds = K + (check ? 1 : 0);
    for (int k = 0; k < rounds; ++k) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) best = max(best, key[i]);
        best = __reduce_max_sync(FULL, best);
        int at = N;
#pragma unroll
        for (int i = V - 1; i >= 0; --i)
            if (key[i] == best) at = lane + 32 * i;
        at = __reduce_min_sync(FULL, at);
        if (check && best != 0u) {
            const float cur = unordered(best);
            if (k > 0 && cur > -INFINITY) {
                const float prev = unordered(before);
                if (prev - cur <= tol + 1.2e-7f * (fabsf(prev) + fabsf(cur))) close = true;
            }
            before = best;
        }
        if (k == lane && k < K) win = at;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane + 32 * i == at) key[i] = 0u;
    }
    if (close) {   // warp-uniform
        __syncwarp();
        win = slow_row<SIGMOID, PAIR>(a, l, shd, lane);
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
        const float y = SIGMOID ? fminf(x, 0.0f) : x;
        const float M = unordered(__reduce_max_sync(FULL, ordered(y)));
        if (has) {
            g = y == M ? 1.0f : expf(y - M);
            if (SIGMOID) g /= 1.0f + expf(-fabsf(x));
        }
        const float s = warp_add(g);
        g = s > 0.0f ? g / s : 0.0f;
    } else if (has) {
        g = SIGMOID ? 1.0f / (1.0f + expf(-x)) : (x == m ? 1.0f : expf(x - m)) * inv;
    }
    if (lane < K) {
        a.idx[(size_t)t * K + lane] = win;
        a.gate[(size_t)t * K + lane] = a.scale * g;
    }
}

template <bool SIGMOID, bool PAIR>
spice_status launch_route_scored(const RouteArgs &a, cudaStream_t st) {
    const unsigned grid = ((unsigned)a.T + WARPS - 1) / WARPS;
    const size_t smem = (size_t)WARPS * a.N * sizeof(double);   // at most 32 KB
    const int v = (a.N + 31) / 32;
    if (v <= 2) route_scored_kernel<2, SIGMOID, PAIR><<<grid, WARPS * 32, smem, st>>>(a);
    else if (v <= 4) route_scored_kernel<4, SIGMOID, PAIR><<<grid, WARPS * 32, smem, st>>>(a);
    else if (v <= 8) route_scored_kernel<8, SIGMOID, PAIR><<<grid, WARPS * 32, smem, st>>>(a);
    else if (v <= 16) route_scored_kernel<16, SIGMOID, PAIR><<<grid, WARPS * 32, smem, st>>>(a);
    else route_scored_kernel<32, SIGMOID, PAIR><<<grid, WARPS * 32, smem, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? SPICE_OK : SPICE_ERR_CUDA;
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
    const RouteArgs a{logits, bias, idx, gate, T, n_experts, top_k, n_groups, top_groups, norm_topk,
                      size > 1 ? (uint32_t)((0x100000000ull + size - 1) / size) : 0u, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool pair = n_groups > 1 && group_score == SPICE_GROUP_TOP2;
    if (score == SPICE_SCORE_SIGMOID) return pair ? launch_route_scored<true, true>(a, st) : launch_route_scored<true, false>(a, st);
    return pair ? launch_route_scored<false, true>(a, st) : launch_route_scored<false, false>(a, st);
}
