// Rows in 8-bit integers: the residual addition with its root-mean-square norm (the step between two layers of the
// stack), and the quantiser of bf16 rows (weights once, SwiGLU activations every step).
//
//   s = bf16(x + delta), x <- s;   p_j = s_j * w_j,   r = 1 / sqrt(mean_j s_j^2 + eps),   h_j = bf16(p_j * r)
//   m = max_j |p_j|;   q_j = 127 p_j / m to the nearest integer, ties to even;   scale = m * r / 127
//
// (the quantiser: p = w, r = 1, no h).  r cancels out of q, and p is a product of two bf16 values, exact in fp32 where it is
// 2^-133 at least (16 significant bits), so the codes are a function of exactly known numbers.  They are rounded exactly: where
// the fp32 quotient lies within its error of a border k + 1/2, 254 |p_j| and (2k + 1) m are compared, both exact in fp32 (16 +
// 7 and 8 + 16 significant bits).  Rows whose largest product lies outside 2^-100 .. 2^100, or whose squares leave fp32's
// range, are evaluated in fp64, where all of these are exact (rows of the quantiser: m is scaled by a power of two).  No
// implementation that keeps the definition can differ by a step.
//
// Both are bound by the bytes that cross HBM (9 per element of a bf16 step with both outputs, 3 for the quantiser): every
// row is read once, held in registers as the packed bf16 pairs it is stored as, and written once (4096 x 2048 with both outputs
// 13.0 us, 0.88 of the measured copy rate; 40960 x 3584 quantised 65 us, 1.04).
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
    float eps, inv_d;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&b);
}

// What turns the values of a row with largest magnitude m into codes
template <bool CHECK>
struct CodeScale {
    float m, c;   // c = 127 / m, within 2^-23 or (without CHECK) rounded up; 0 where m is not well inside fp32's range
    __device__ __forceinline__ explicit CodeScale(float largest) {
        m = largest;
        c = 0.0f;
        if (CHECK) {   // (m is well inside)
            c = __fdividef(1.0f, m);
            c = 127.0f * fmaf(c, fmaf(-m, c, 1.0f), c);
        } else if (m > 0x1p-100f && m < 0x1p100f) {
            c = __fdiv_ru(127.0f, m);
        }
    }
};

// nearest integer to 127 p / m, ties to even, exactly, for |127 p / m| between the integers a and a + 1: both products have
// at most 24 significant bits.
__device__ __forceinline__ float round_at_border(float p, float m, float a, bool odd) {
    const float lhs = 254.0f * fabsf(p), rhs = (2.0f * a + 1.0f) * m;
    return copysignf(a + (lhs > rhs || (lhs == rhs && odd) ? 1.0f : 0.0f), p);
}

// the code of a bf16 value in a row at the ends of fp32's range: m is brought into [1, 2) by a power of two first
__device__ __noinline__ float code_scaled(float p, float m) {
    if (!(m > 0.0f)) return 0.0f;
    const int e = (int)(__float_as_uint(m) >> 23);                                    // biased exponent
    const float f = __uint_as_float((uint32_t)min(max(254 - e, 1), 253) << 23);       // 2^(127 - e): at most 2^126
    const float mn = m * f, pn = p * f;
    const float u = pn * (127.0f / mn);
    const float k = rintf(u);
    const float a = floorf(fabsf(u));
    return fabsf(u - k) > 0.4999f ? round_at_border(pn, mn, a, (int)a & 1) : k;
}

// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Codes of 8 values as packed bytes.  p c + 1.5 * 2^23 in one rounding is the nearest integer to p c, its low byte the code.
// CHECK (products of two bf16): p c is off by at most 127 * 2^-23 < 1.6e-5 from the quotient; where one of the values lies
// within 2e-5 of a border they are looked at once more.
// Without (bf16 values): the answer is exact as it is.  With p = P 2^t, m = M and integers 128 <= P, M < 256, the quotient
// 127 P 2^t / M is at least 2^t / (2 M) > 2^t * 0.0019 away from every border it does not lie on, and p c is off by
// 2^t * 3.1e-5 at most.  It lies on a border only where 254 P 2^t = (2 k + 1) M: 127 then divides M, c is a power of two
// and p c exact, or 127 divides 2 k + 1, the border is 63.5 (half of the row's largest, a frequent value), and c, rounded
// up, takes it to 64, the even side.
template <bool CHECK>
__device__ __forceinline__ uint2 codes_of(const float (&p)[8], const CodeScale<CHECK> &c) {
    constexpr float MAGIC = 12582912.0f;
    uint32_t k[8];
    float off = CHECK || c.c > 0.0f ? 0.0f : 1.0f;
    const uint64_t c2 = pair2(c.c, c.c), magic2 = pair2(MAGIC, MAGIC), minus2 = pair2(-1.0f, -1.0f);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const uint64_t p2 = pair2(p[j], p[j + 1]);
        const uint64_t s2 = fma2(p2, c2, magic2);
        if (CHECK) {
            const uint64_t d2 = fma2(p2, c2, fma2(s2, minus2, magic2));
            off = fmaxf(off, fabsf(__uint_as_float((uint32_t)d2)));
            off = fmaxf(off, fabsf(__uint_as_float((uint32_t)(d2 >> 32))));
        }
        k[j] = (uint32_t)s2;
        k[j + 1] = (uint32_t)(s2 >> 32);
    }
    if (off > 0.49998f) {
        if (CHECK) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = __uint_as_float(k[j]) - MAGIC;      // the nearest integer; the other side of the border is n +- 1
                const float d = __fmaf_rn(p[j], c.c, -n);
                if (fabsf(d) > 0.49998f) {
                    const bool outer = n != 0.0f && (d > 0.0f) != (n > 0.0f);   // n is the one further from 0
                    k[j] = __float_as_uint(round_at_border(p[j], c.m, fabsf(n) - (outer ? 1.0f : 0.0f), ((k[j] & 1u) != 0u) != outer) + MAGIC);
                }
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                float v = p[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) v = i == j ? p[i] : v;
                const uint32_t code = __float_as_uint(code_scaled(v, c.m) + MAGIC);
#pragma unroll
                for (int i = 0; i < 8; ++i) k[i] = i == j ? code : k[i];
            }
        }
    }
    const uint32_t a = __byte_perm(k[0], k[1], 0x0040), b = __byte_perm(k[2], k[3], 0x0040);
    const uint32_t d = __byte_perm(k[4], k[5], 0x0040), e = __byte_perm(k[6], k[7], 0x0040);
    return make_uint2(__byte_perm(a, b, 0x5410), __byte_perm(d, e, 0x5410));
}

// the larger magnitude; a NaN on either side stays
__device__ __forceinline__ float max_abs_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}

__device__ __forceinline__ float warp_sum_xor(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ double warp_sum_xor(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_max_xor(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// A row whose squares or products come near the ends of fp32's range, in fp64, where both are exact: the scale, the codes and
// h (the stream is written already).  Such rows are rare, so the row is read again, by the threads that wrote it; nothing of it
// is kept in registers.  The quotient 127 p / m is at least 2^-27 away from a border that it does not lie on (16 significant
// bits in p and m, and p > m / 256 where a border is near), so its rounding to fp64 crosses none.  zeros: the row has nothing
// but zeros, as the rows that fill up a batch.
template <bool WIDE>
__device__ __noinline__ void row_in_fp64(const RowArgs a, size_t row, int i0, int step, bool zeros) {
    __shared__ double sh_sum[32], sh_top[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    const int nv = a.d >> 3;
    const size_t base = row * (size_t)a.d;
    auto word_x = [&](int i, int j) { return reinterpret_cast<const uint32_t *>(a.x + base)[i * 4 + j]; };
    auto word_w = [&](int i, int j) { return reinterpret_cast<const uint32_t *>(a.weight)[i * 4 + j]; };
    if (zeros) {   // 64 rows of 2048: 2.1 us, 4.4 by way of what follows
        if (a.q && i0 == 0) a.scale[row] = 1.0f;
        for (int i = i0; i < nv; i += step) {
#pragma unroll 1
            for (int j = 0; j < 4; ++j)
                if (a.h) reinterpret_cast<uint32_t *>(a.h + base)[i * 4 + j] = (word_x(i, j) ^ word_w(i, j)) & 0x80008000u;
            if (a.q) *reinterpret_cast<uint2 *>(a.q + base + (size_t)i * 8) = make_uint2(0u, 0u);
        }
        return;
    }
    double sum = 0.0, top = 0.0;
    for (int i = i0; i < nv; i += step) {
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
            const uint32_t x = word_x(i, k >> 1), w = word_w(i, k >> 1);
            const double s = k & 1 ? bf_hi(x) : bf_lo(x), p = s * (double)(k & 1 ? bf_hi(w) : bf_lo(w));
            sum += s * s;
            top = fmax(top, p == p ? fabs(p) : (double)INFINITY);
        }
    }
    sum = warp_sum_xor(sum);
    top = warp_max_xor(top);
    if (WIDE) {
        if (lane == 0) {
            sh_sum[warp] = sum;
            sh_top[warp] = top;
        }
        __syncthreads();
        sum = warp_sum_xor(lane < nw ? sh_sum[lane] : 0.0);
        top = warp_max_xor(lane < nw ? sh_top[lane] : 0.0);
    }
    const double r = 1.0 / sqrt(sum / a.d + (double)a.eps);
    const bool codes = (float)top < INFINITY && ((float)r < INFINITY || top == 0.0);
    if (a.q && i0 == 0) a.scale[row] = !codes ? __uint_as_float(0x7fffffffu) : top == 0.0 ? 1.0f : (float)(top * r / 127.0);
    for (int i = i0; i < nv; i += step) {
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
            const uint32_t x = word_x(i, k >> 1), w = word_w(i, k >> 1);
            const double p = (double)(k & 1 ? bf_hi(x) : bf_lo(x)) * (double)(k & 1 ? bf_hi(w) : bf_lo(w));
            const size_t at = base + (size_t)i * 8 + k;
            if (a.h) a.h[at] = __float2bfloat16_rn((float)(p * r));
            if (a.q) a.q[at] = codes && top > 0.0 ? (int8_t)(int)rint(127.0 * p / top) : (int8_t)0;
        }
    }
}

// threads of a block: what its registers leave room for
template <int V>
constexpr int most_threads() {
    return V <= 2 ? 1024 : 512;
}

// One row per group of threads: a warp (WIDE = false, several rows per block) or the whole block.  A thread holds V
// vectors of 8 elements, `step` threads apart.
template <int V, int MODE, bool WIDE>
__global__ void __launch_bounds__(WIDE ? most_threads<V>() : 256) rows_i8_kernel(const RowArgs a, const size_t rows) {
    __shared__ float sh_sum[32];
    __shared__ uint32_t sh_max[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nw = blockDim.x >> 5;
    const size_t row = WIDE ? blockIdx.x : (size_t)blockIdx.x * nw + warp;
    grid_dependency();
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

    constexpr bool KEEP = MODE != NO_NORM && V <= 2;   // the products stay in registers
    float kept[KEEP ? V : 1][8];
    float sum = 0.0f;
    float top = 0.0f;       // largest |p|
    uint32_t top16 = 0;     // NO_NORM: the same of the bits of two bf16 at a time (they order like the values)
#pragma unroll
    for (int v = 0; v < V; ++v) {
        uint32_t *x = reinterpret_cast<uint32_t *>(&xs[v]);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&wt[MODE != NO_NORM ? v : 0]);
        const uint32_t *d16 = reinterpret_cast<const uint32_t *>(&dl[MODE == DELTA_BF16 ? v : 0]);
        const float *d32 = reinterpret_cast<const float *>(&df[MODE == DELTA_F32 ? 2 * v : 0]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (MODE == DELTA_BF16) {   // (a sum of two bf16 rounds to bf16 the same directly and by way of fp32)
                const __nv_bfloat162 s = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&x[j]),
                                                 *reinterpret_cast<const __nv_bfloat162 *>(&d16[j]));
                x[j] = *reinterpret_cast<const uint32_t *>(&s);
            }
            if (MODE == DELTA_F32) x[j] = pack_bf16(bf_lo(x[j]) + d32[2 * j], bf_hi(x[j]) + d32[2 * j + 1]);
            const float lo = bf_lo(x[j]), hi = bf_hi(x[j]);
            if (MODE == NO_NORM) {
                top16 = __vmaxu2(top16, x[j] & 0x7fff7fffu);
            } else {
                sum = fmaf(lo, lo, sum);
                sum = fmaf(hi, hi, sum);
                const float p0 = lo * bf_lo(w[j]), p1 = hi * bf_hi(w[j]);
                top = max_abs_nan(top, p0);
                top = max_abs_nan(top, p1);
                if (KEEP) {
                    kept[KEEP ? v : 0][2 * j] = p0;
                    kept[KEEP ? v : 0][2 * j + 1] = p1;
                }
            }
        }
        const int i = i0 + v * step;
        if ((MODE == DELTA_BF16 || MODE == DELTA_F32) && i < nv) *reinterpret_cast<uint4 *>(a.x + base + (size_t)i * 8) = xs[v];
    }
    // as bits: magnitudes order like integers, infinities and NaN on top
    uint32_t big = MODE == NO_NORM ? max(top16 << 16, top16 & 0xffff0000u) : __float_as_uint(top) & 0x7fffffffu;
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
    const float m = __uint_as_float(big);
    float r = 1.0f;
    if (MODE != NO_NORM) {
        const float mean = sum * a.inv_d + a.eps;
        // (the same for the whole row; a NaN compares false.  r <= 2^23: a product below fp32's range, off by 2^-150, moves h by
        // less than the smallest normal number)
        if (!(m > 0x1p-100f && m < 0x1p100f && mean >= 0x1p-46f && mean < INFINITY)) {
            uint32_t any = m == 0.0f && mean >= 0x1p-46f ? 0u : 1u;
#pragma unroll
            for (int v = 0; v < V; ++v) any |= (xs[v].x | xs[v].y | xs[v].z | xs[v].w) & 0x7fff7fffu;
            any = WIDE ? __syncthreads_or(any != 0u) : __any_sync(0xffffffffu, any != 0u);
            row_in_fp64<WIDE>(a, row, i0, step, any == 0u);
            return;
        }
        r = rsqrtf(mean);
        r = r * (1.5f - 0.5f * mean * r * r);   // (one Newton step: within an ulp)
    }
    const bool finite = MODE != NO_NORM || big < 0x7f800000u;
    if (a.q && i0 == 0) {
        constexpr float C = 1.0f / 127.0f;
        a.scale[row] = !finite ? __uint_as_float(0x7fffffffu) : m == 0.0f ? 1.0f : m > 1.0f ? (m * C) * r : m * (r * C);
    }
    const CodeScale<MODE != NO_NORM> cs(finite ? m : 0.0f);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = i0 + v * step;
        if (i >= nv) break;
        const uint32_t *x = reinterpret_cast<const uint32_t *>(&xs[v]);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&wt[MODE != NO_NORM ? v : 0]);
        float p[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p[2 * j] = KEEP ? kept[KEEP ? v : 0][2 * j] : MODE == NO_NORM ? bf_lo(x[j]) : bf_lo(x[j]) * bf_lo(w[j]);
            p[2 * j + 1] = KEEP ? kept[KEEP ? v : 0][2 * j + 1] : MODE == NO_NORM ? bf_hi(x[j]) : bf_hi(x[j]) * bf_hi(w[j]);
        }
        if (MODE != NO_NORM && a.h)
            *reinterpret_cast<uint4 *>(a.h + base + (size_t)i * 8) = make_uint4(pack_bf16(p[0] * r, p[1] * r), pack_bf16(p[2] * r, p[3] * r),
                                                                              pack_bf16(p[4] * r, p[5] * r), pack_bf16(p[6] * r, p[7] * r));
        if (a.q) *reinterpret_cast<uint2 *>(a.q + base + (size_t)i * 8) = finite ? codes_of<MODE != NO_NORM>(p, cs) : make_uint2(0u, 0u);
    }
}

constexpr int MAX_COLS = 32768;   // 512 threads x 8 vectors x 8 elements: what a block holds in registers

template <int MODE>
spice_status launch_rows(const RowArgs &a, size_t rows, cudaStream_t st) {
    const int nv = a.d >> 3;
    bool ok = false;
    auto wide = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int threads = ((nv + V - 1) / V + 31) & ~31;
        ok = launch_early(rows_i8_kernel<V, MODE, true>, dim3((unsigned)rows), threads, 0, st, 1, a, rows);
    };
    auto narrow = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int wpb = rows < 8 * 296 ? 4 : 8;
        ok = launch_early(rows_i8_kernel<V, MODE, false>, dim3((unsigned)((rows + wpb - 1) / wpb)), wpb * 32, 0, st, 1, a, rows);
    };
    using std::integral_constant;
    // Few rows: a vector per thread, the shortest chain.  Many: more per thread, so that what a thread does beside its data
    // (reductions, the row's scale) is spread over more of it, as long as enough warps stay resident.
    // Norm with 1 / 2 vectors: 16 rows of 2048 1.6 / 1.8 us, 4096 rows of 2048 13.8 / 13.0.  Quantiser with 1 / 2 / 4: 40960 rows
    // of 3584 111 / 90 / 65, 333 rows of 2816 2.5 each.  (Eight: what a row of more than 16384 takes; 2048 rows of 20480 67.)
    const bool many = rows >= 1024;
    if (nv <= 32) narrow(integral_constant<int, 1>{});
    else if (nv <= 64) narrow(integral_constant<int, 2>{});
    else if (!many && nv <= 1024) wide(integral_constant<int, 1>{});
    else if (nv > 2048) wide(integral_constant<int, 8>{});
    else if constexpr (MODE == NO_NORM) {
        if (many) wide(integral_constant<int, 4>{});
        else wide(integral_constant<int, 2>{});
    } else {
        wide(integral_constant<int, 2>{});
    }
    return ok ? SPICE_OK : SPICE_ERR_CUDA;
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
                    reinterpret_cast<const __nv_bfloat16 *>(weight), reinterpret_cast<__nv_bfloat16 *>(h), q, scale, d, eps, 1.0f / (float)d};
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
                    q, scale, cols, 0.0f, 0.0f};
    return launch_rows<NO_NORM>(a, (size_t)rows, static_cast<cudaStream_t>(stream));
}
