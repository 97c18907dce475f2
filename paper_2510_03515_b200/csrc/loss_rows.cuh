// What the losses of rapid_losses.h share: the scratch, the statistics of a row of logits and the gradient of a row.
//
// All three losses have the same shape.  A row r of logits z gives a log-sum-exp of z / tau; an operator turns it, together with
// a few chosen columns of the row, into a factor a_r and values for those columns; the gradient is
//     dz[v] = a_r softmax(z / tau)_v  everywhere else,   dz[column_j] = value_j.
// An operator says what the chosen columns are (the sampled token, or a teacher's list) and computes the factor and the values,
// in double, with one warp; this file and loss_rows.cu do the rest.
//
// Logarithms are base 2 inside: x_v = z_v log2(e) / tau, lse2 = log2 sum_v 2^(x_v).
#pragma once

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rapid_common.cuh"
#include "rapid_losses.h"

namespace rapid {
namespace losses {

static_assert(sizeof(rapid_clip_desc_t) == 80 && sizeof(rapid_pref_desc_t) == 80 && sizeof(rapid_distill_desc_t) == 72 &&
                  sizeof(rapid_loss_stats_t) == 48,
              "bindings rely on these");

constexpr int kMaxList = 256;      // entries of a distillation list
constexpr int kPrepBlocks = 1024;  // blocks of a preparing kernel, at most
constexpr int kSumBlocks = 1024;   // blocks of a summing kernel, at most
constexpr int64_t kMaxRows = 0x7fffffffll - 1023;  // a position plus a block's threads stays within 31 bits

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t elem_size(int32_t dtype) { return dtype == RAPID_BF16 ? 2 : 4; }

// ---- scratch ------------------------------------------------------------------------------------------------

struct Header {
    unsigned int ticket;  // rows handed out
    unsigned int done;    // blocks of the summing kernel that are through
    int32_t status;       // RAPID_ERR_TIMEOUT when a wait gave up
    int32_t pad;
};

// A warp's part of a row: its largest logit m, its shift sh and s, the sum of its 2^(x_v - sh).
struct WarpPart {
    double s;
    float m, sh;  // sh = -inf where there is nothing
};

struct Scratch {
    Header* head;
    int2* counts;         // [kPrepBlocks] rows that count, rows that are not valid
    double* sums;         // [kSumBlocks][8] partial sums
    double* lse2;         // [T]
    double* value;        // [T] log-probability of the token, or the row's loss
    float* row_max;       // [T]
    uint8_t* state;       // [T] ROW_*
    int32_t* seq_rows;    // [N] rows that count
    int32_t* seq_bad;     // [N] rows that are not valid
    double* seq_sum;      // [N] s_n
    double* seq_coef;     // [N] g_n
    unsigned long long* seq_top;  // [N] the largest slope of its pairs, where there are many
    double* pair_slope;   // [P]
    double* teacher_lse2; // [T]
    WarpPart* parts;      // [T][pieces] of rows that are read without a gradient
    float* token_z;       // [T] the token's logit
};

enum : int { NEED_SEQ = 1, NEED_PAIRS = 2, NEED_TEACHER = 4 };

// Warps that share a row that is read without a gradient: 1024 vectors for each at the least, four at most (with as many as there are
// 1024 vectors, 19 on 151936 bf16 columns, 8192 rows take 896 us instead of 838).
inline int stat_pieces(int32_t vocab, int32_t dtype) {
    const int64_t n = (vocab / (16 / (int64_t)elem_size(dtype)) + 1023) / 1024;
    return n < 1 ? 1 : n > 4 ? 4 : (int)n;
}

// Vectors of a piece of a row whose gradient is written by token_grads_kernel, and such pieces of a row.
constexpr int kPieceVecs = 16 * 32;
inline int64_t grad_pieces(int32_t vocab, int32_t dtype) {
    const int64_t n = (vocab / (16 / (int64_t)elem_size(dtype)) + kPieceVecs - 1) / kPieceVecs;
    return n < 1 ? 1 : n;
}

// Carve `base` (256-byte aligned); returns the bytes used.
inline size_t carve(int64_t T, int64_t N, int64_t P, int pieces, int need, void* base, Scratch* out) {
    size_t off = 0;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* q = p ? p + off : nullptr;
        off = align_up(off + bytes, 256);
        return q;
    };
    Scratch s{};
    s.head = reinterpret_cast<Header*>(take(sizeof(Header)));
    s.counts = reinterpret_cast<int2*>(take(kPrepBlocks * sizeof(int2)));
    s.sums = reinterpret_cast<double*>(take((size_t)kSumBlocks * 64));
    s.lse2 = reinterpret_cast<double*>(take((size_t)T * 8));
    s.value = reinterpret_cast<double*>(take((size_t)T * 8));
    s.row_max = reinterpret_cast<float*>(take((size_t)T * 4));
    s.state = reinterpret_cast<uint8_t*>(take((size_t)T));
    if (need & NEED_SEQ) s.seq_rows = reinterpret_cast<int32_t*>(take((size_t)N * 4));
    if (need & NEED_PAIRS) {
        s.seq_bad = reinterpret_cast<int32_t*>(take((size_t)N * 4));
        s.seq_sum = reinterpret_cast<double*>(take((size_t)N * 8));
        s.seq_coef = reinterpret_cast<double*>(take((size_t)N * 8));
        s.seq_top = reinterpret_cast<unsigned long long*>(take((size_t)N * 8));
        s.pair_slope = reinterpret_cast<double*>(take((size_t)P * 8));
    }
    if (need & NEED_TEACHER) s.teacher_lse2 = reinterpret_cast<double*>(take((size_t)T * 8));
    if (pieces > 0) {
        s.parts = reinterpret_cast<WarpPart*>(take((size_t)T * pieces * sizeof(WarpPart)));
        s.token_z = reinterpret_cast<float*>(take((size_t)T * 4));
    }
    if (out) *out = s;
    return off;
}

// ---- host checks that all three share --------------------------------------------------------------------------

// Do two matrices of `n` rows, `width` bytes wide at pitches of pa and pb bytes, share a byte?  Matrices of one pitch may lie side
// by side in the same rows; of two pitches, they have to be apart altogether.
inline bool matrices_overlap(const void* a, int64_t pa, const void* b, int64_t pb, int64_t n, int64_t width) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    const size_t ea = (size_t)(n - 1) * pa + width, eb = (size_t)(n - 1) * pb + width;
    if (x >= y + eb || y >= x + ea) return false;
    if (pa != pb) return true;
    int64_t off = ((int64_t)y - (int64_t)x) % pa;
    if (off < 0) off += pa;
    return off < width || off + width > pa;
}

inline rapid_status_t check_shape(int64_t T, int32_t vocab, int32_t dtype, int64_t ld, int64_t ld_grad, uint32_t flags, uint32_t known,
                                  double scale, double norm_z) {
    if (T <= 0 || vocab <= 0 || ld < vocab || ld_grad < vocab) return RAPID_ERR_INVALID_ARG;
    if (dtype != RAPID_F32 && dtype != RAPID_BF16) return RAPID_ERR_INVALID_ARG;
    if ((flags & ~known) || !isfinite(scale)) return RAPID_ERR_INVALID_ARG;
    if ((flags & RAPID_LOSS_NORM_GIVEN) && !(norm_z > 0.0 && isfinite(norm_z))) return RAPID_ERR_INVALID_ARG;
    // 2^56 elements are far beyond any device's memory; keeps every offset of an element in 64 bits
    if (T > kMaxRows || vocab > (1 << 30) || ld > (1ll << 56) / T || ld_grad > (1ll << 56) / T) return RAPID_ERR_UNSUPPORTED;
    const size_t es = elem_size(dtype);
    if ((size_t)ld * es % 16 != 0 || (size_t)ld_grad * es % 16 != 0) return RAPID_ERR_ALIGNMENT;
    return RAPID_OK;
}

inline rapid_status_t check_matrices(const void* logits, const void* dlogits, int64_t T, int32_t vocab, int32_t dtype, int64_t ld,
                                     int64_t ld_grad) {
    if (!logits) return RAPID_ERR_INVALID_ARG;
    if (!aligned(logits, 16) || !aligned(dlogits, 16)) return RAPID_ERR_ALIGNMENT;
    if (!dlogits) return RAPID_OK;
    const int64_t es = (int64_t)elem_size(dtype);
    if (logits == dlogits) return ld == ld_grad || T == 1 ? RAPID_OK : RAPID_ERR_INVALID_ARG;
    return matrices_overlap(logits, ld * es, dlogits, ld_grad * es, T, vocab * es) ? RAPID_ERR_INVALID_ARG : RAPID_OK;
}

// sm_100 only.  Returns the SM count of the current device through *sm_count.
inline rapid_status_t check_device(int* sm_count) {
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return RAPID_ERR_CUDA;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(sm_count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return RAPID_ERR_CUDA;
    return major == 10 ? RAPID_OK : RAPID_ERR_UNSUPPORTED;
}

// ---- a row's statistics -----------------------------------------------------------------------------------------

// log2(e) / tau, as a sum of two floats: k1, cut after some bits, and k2 > 0 with the next 24 (k2 is never 0, or -inf * k2 would be NaN).
// bf16: 16 bits, so that the product with a logit (8 bits) and its difference from the shift are exact, and the argument is rounded once.
// float: 24, as it is rounded twice anyhow; the first time at the size of z k2, which for logits far from 0 has to be small (with 16
// a log-sum-exp is off by 1e-4 at |z| / tau of 2^27).  `rest` is ln(2) times what the two leave of kd: it is the same for all terms of a size,
// so their sum is put right.  k is the nearest float.
struct Factor {
    double kd, rest;
    float k1, k2, k;
};
inline Factor make_factor(double tau, int32_t dtype) {
    const int bits = dtype == RAPID_BF16 ? 16 : 24;
    Factor f;
    f.kd = kLog2eD / tau;
    int e = 0;
    const double m = frexp(f.kd, &e);  // in [1/2, 1)
    f.k1 = (float)ldexp(floor(ldexp(m, bits)), e - bits);
    f.k2 = (float)(f.kd - (double)f.k1);
    if (!(f.k2 > 0.f)) f.k2 = 1e-30f;
    f.rest = (f.kd - ((double)f.k1 + (double)f.k2)) * kLn2D;
    f.k = (float)f.kd;
    return f;
}

// Division of a number below 2^31 by one that is known on the host: the high word of a product (Granlund and Montgomery).
struct Divisor {
    uint32_t by, times, shift;
};
inline Divisor make_divisor(int32_t d) {
    Divisor v{(uint32_t)d, 0u, 0u};
    while ((1ll << v.shift) < d) ++v.shift;
    v.times = (uint32_t)(((1ull << (31 + v.shift)) + d - 1) / (uint64_t)d);  // below 2^32 for d >= 2, as 2^shift < 2 d
    return v;
}

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t divide(int64_t n, const Divisor& d) {
    return d.by == 1 ? (uint32_t)n : __umulhi((uint32_t)n, d.times) >> (d.shift - 1);
}

template <int DT>
struct Elem;
template <>
struct Elem<RAPID_BF16> {
    using T = uint16_t;
    static constexpr int kPer = 8;  // elements of a 16-byte vector
    __device__ static __forceinline__ float get(T x) { return __uint_as_float((uint32_t)x << 16); }
    __device__ static __forceinline__ T put(float x) { return (T)(pack_bf16x2(x, 0.f) & 0xffffu); }
    __device__ static __forceinline__ float largest(const uint4& q) {
        const uint32_t m = bf16x2_max(bf16x2_max(q.x, q.y), bf16x2_max(q.z, q.w));
        return fmaxf(bf16_lo(m), bf16_hi(m));
    }
    // the i-th pair of elements
    __device__ static __forceinline__ uint64_t pair(const uint4& q, int i) {
        const uint32_t w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
        return f32x2(bf16_lo(w), bf16_hi(w));
    }
};
template <>
struct Elem<RAPID_F32> {
    using T = float;
    static constexpr int kPer = 4;
    __device__ static __forceinline__ float get(T x) { return x; }
    __device__ static __forceinline__ T put(float x) { return x; }
    __device__ static __forceinline__ float largest(const uint4& q) {
        return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    __device__ static __forceinline__ uint64_t pair(const uint4& q, int i) {
        return i == 0 ? f32x2(__uint_as_float(q.x), __uint_as_float(q.y)) : f32x2(__uint_as_float(q.z), __uint_as_float(q.w));
    }
};

// Mean relative error of the hardware exponential over the fraction of its argument (errors lie in [-1.44e-7, +0.63e-7]; measured
// over all 2^23 fractions): a sum of many terms carries it and is divided by 1 + kEx2Mean.
constexpr float kEx2Mean = -4.95e-8f;
constexpr float kNothing = -1.0e38f;  // at or below: -inf or the lowest finite value, a masked part of the vocabulary

// Both halves of a packed pair of bf16 values, each with a float added to it, in one instruction each.
__device__ __forceinline__ uint64_t bf16x2_plus(uint32_t p, float b) {
    float lo, hi;
    asm("{\n\t.reg .b16 l, h;\n\t"
        "mov.b32 {l, h}, %2;\n\t"
        "add.rn.f32.bf16 %0, l, %3;\n\t"
        "add.rn.f32.bf16 %1, h, %3;\n\t}"
        : "=f"(lo), "=f"(hi)
        : "r"(p), "f"(b));
    return f32x2(lo, hi);
}

// One thread's part of a row: the largest logit m, the shift sh that its exponentials are taken against, and sum_v 2^(x_v - sh)
// with the rounding errors of its additions beside it.  sh = ceil(m k) + off is used as it stands, here and where the parts meet,
// so no rounding of m k enters; `off`, a 16-bit fraction, is one for a warp (the parts of its lanes differ by exact powers of two)
// and another for each warp, so that the errors of the exponentials of equal logits do not all have one sign.
struct Part {
    float m = -INFINITY, sh = 0.f, s = 0.f, c = 0.f;

    __device__ __forceinline__ void see(float bm, float off, const Factor& f) {
        if (bm > m) {
            m = bm;
            if (bm > kNothing) {
                const float now = ceilf(bm * f.k) + off;
                const float by = ex2_approx(sh - now);  // an exact power of two; of an empty part, whatever: its sum is 0
                if (s > 0.f) {
                    s *= by;
                    c *= by;
                }
                sh = now;
            }
        }
    }
    __device__ __forceinline__ void add(float b) {  // Fast2Sum wants the larger one first
        const float hi = fmaxf(s, b), lo = fminf(s, b);
        const float t = hi + lo;
        c += (hi - t) + lo;
        s = t;
    }
    __device__ __forceinline__ float term(float z, const Factor& f) const { return ex2_approx(fmaf(z, f.k2, fmaf(z, f.k1, -sh))); }

    // U vectors: the exponentials are summed from zero, in as many partial sums as a vector has elements, and then added
    template <int DT, int U>
    __device__ __forceinline__ void vectors(const uint4 (&q)[U], float off, const Factor& f) {
        constexpr int P = Elem<DT>::kPer / 2;
        float bm = Elem<DT>::largest(q[0]);
#pragma unroll
        for (int j = 1; j < U; ++j) bm = fmaxf(bm, Elem<DT>::largest(q[j]));
        see(bm, off, f);
        const uint64_t k1 = f32x2(f.k1, f.k1), k2 = f32x2(f.k2, f.k2), nsh = f32x2(-sh, -sh);
        uint64_t a[P];
#pragma unroll
        for (int i = 0; i < P; ++i) a[i] = f32x2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < U; ++j) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const uint64_t z = Elem<DT>::pair(q[j], i);
                float x0, x1;
                f32x2_split(f32x2_fma(z, k2, f32x2_fma(z, k1, nsh)), x0, x1);
                a[i] = f32x2_add(a[i], f32x2(ex2_approx(x0), ex2_approx(x1)));
            }
        }
#pragma unroll
        for (int n = P / 2; n > 0; n /= 2)
#pragma unroll
            for (int i = 0; i < n; ++i) a[i] = f32x2_add(a[i], a[i + n]);
        float s0, s1;
        f32x2_split(a[0], s0, s1);
        add(s0 + s1);
    }
    __device__ __forceinline__ void scalar(float z, float off, const Factor& f) {
        see(z, off, f);
        if (z > kNothing) add(term(z, f));
    }
};

// 2^y and log2(s) in double where a whole row waits for them: Taylor's series of e^t for |t| <= ln(2) / 2 to t^11 (the rest is below
// 7e-15) evaluated in pairs, six dependent steps; the logarithm by one step of Newton's iteration from the hardware's.  No
// branch for far arguments: the calls are inlined some ten times in a kernel whose warps are at different places of it, and what they
// take in the instruction cache counts (with a call of exp2() for those 65536 x 4096 distillation rows took 215 us, without 194).
__device__ __forceinline__ double exp2_short(double y) {
    const double in = y < -2100.0 ? -2100.0 : y > 2100.0 ? 2100.0 : y;
    // the nearest whole number by adding 1.5 2^52, in whose low word it then stands: no conversion, which would be a slow one
    const double up = in + 6755399441055744.0, n = up - 6755399441055744.0;
    const double t = (in - n) * kLn2D, t2 = t * t, t4 = t2 * t2;
    const double a0 = 1.0 + t, a1 = fma(t, 1.0 / 6, 0.5), a2 = fma(t, 1.0 / 120, 1.0 / 24), a3 = fma(t, 1.0 / 5040, 1.0 / 720);
    const double a4 = fma(t, 1.0 / 362880, 1.0 / 40320), a5 = fma(t, 1.0 / 39916800, 1.0 / 3628800);
    const double b0 = fma(a1, t2, a0), b1 = fma(a3, t2, a2), b2 = fma(a5, t2, a4);
    // 2^n in two factors, the last of which overflows or underflows where the result does (of NaN, t is NaN)
    const int e = __double2loint(up), half = e >> 1, rest = e - half;
    const double lo = __hiloint2double((min(max(half, -1022), 1023) + 1023) << 20, 0), hi = __hiloint2double((min(max(rest, -1022), 1023) + 1023) << 20, 0);
    return fma(b2, t4 * t4, fma(b1, t4, b0)) * lo * hi;
}
__device__ __forceinline__ double log2_short(double s) {  // s > 0, normal
    const int e = (__double2hiint(s) >> 20) - 1023;
    const double m = __hiloint2double(__double2hiint(s) - (e << 20), __double2loint(s));  // in [1, 2)
    const float near = __uint_as_float(0x3f800000u | ((uint32_t)__double2hiint(m) & 0xfffffu) << 3 | (uint32_t)__double2loint(m) >> 29);  // m cut to a float
    const double l = (double)__log2f(near);
    const double r = fma(m, exp2_short(-l), -1.0);  // below 1e-6
    return (double)e + fma(r * fma(r, -0.5, 1.0), kLog2eD, l);
}

// Sum and maximum over W neighbouring lanes; all of the warp comes here.
template <int W>
__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int W>
__device__ __forceinline__ float lanes_top(float v) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Maximum over the warp of floats that are not NaN.
__device__ __forceinline__ float warp_top(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// A warp's part: 2^sh s is its sum.  The largest term of each lane is taken out and put back in double, without the error of the
// hardware's exponential: where a few logits hold most of a row's sum (2000 logits of standard deviation 3) two of them are hardly ever
// one lane's.  (Of 1600 small calls with sizes drawn at random, 2 had a loss off by more than 3e-7; with the warp's largest alone, 6.)
__device__ __forceinline__ WarpPart warp_part(const Part& p, const Factor& f) {
    WarpPart w;
    w.m = warp_top(p.m);
    w.sh = warp_top(p.s > 0.f ? p.sh : -INFINITY);
    double s = 0.0;
    if (p.s > 0.f) {
        s = ((double)p.s + (double)p.c - (double)p.term(p.m, f)) * fma((double)p.m, f.rest, 1.0 / (1.0 + (double)kEx2Mean)) + exp2_short((double)p.m * f.kd - (double)p.sh);
        s *= (double)ex2_approx(p.sh - w.sh);  // an exact power of two
    }
    w.s = warp_sum(s);
    return w;
}

struct RowStat {
    double lse2;  // -inf when no logit is left
    float max;
};
// The warps' parts together, by one warp, of which lane i holds warp i's.
__device__ __forceinline__ RowStat join_parts(const WarpPart& p) {
    RowStat r{-INFINITY, warp_top(p.m)};
    const float top = warp_top(p.sh);
    const double s = warp_sum(p.sh > -INFINITY ? p.s * exp2_short((double)p.sh - (double)top) : 0.0);
    if (s > 0.0) r.lse2 = (double)top + log2_short(s);
    return r;
}

// The same where one warp has the whole row.
__device__ __forceinline__ RowStat one_part(const WarpPart& p) {
    return RowStat{p.s > 0.0 ? (double)p.sh + log2_short(p.s) : -INFINITY, p.m};
}

// And by one thread, from memory.
__device__ __forceinline__ RowStat stored_parts(const WarpPart* parts, int pieces) {
    RowStat r{-INFINITY, -INFINITY};
    float top = -INFINITY;
    for (int p = 0; p < pieces; ++p) {
        r.max = fmaxf(r.max, parts[p].m);
        top = fmaxf(top, parts[p].sh);
    }
    double s = 0.0;
    for (int p = 0; p < pieces; ++p)
        if (parts[p].sh > -INFINITY) s += parts[p].s * exp2_short((double)parts[p].sh - (double)top);
    if (s > 0.0) r.lse2 = (double)top + log2_short(s);
    return r;
}

__device__ __forceinline__ float shift_fraction(int warp) { return (float)(((unsigned)warp * 40503u) & 0xffffu) * (1.f / 65536.f); }

// ---- a row's gradient --------------------------------------------------------------------------------------------

// dz_v = a 2^(x_v - lse2).  The largest logit m is taken off first, which keeps the argument (z_v - m) k + c small whatever the logits'
// size, and so its rounding below the result's: c is some 2^7 at most, so the argument is off by 2^-18 of a probability.  bf16: |a| goes
// into c too, and an element costs an addition (which widens it as well), a multiply-add and an exponential.  float: a is multiplied at the
// end, but for powers of two above one, which go into c: a factor may be beyond the floats (a ratio of e^90) where its products with small
// probabilities are not, and its product with none is 0.  The constants are formed once a row; the hardware's logarithm is off by 2^-22.
struct RowGrad {
    double a, lse2;
};
struct GradConst {
    float c, m, a;
};
template <int DT>
__device__ __forceinline__ GradConst grad_const(const RowGrad& g, float max, const Factor& f) {
    GradConst k;
    k.m = max > kNothing ? max : 0.f;
    const double a = g.a > 1e300 ? 1e300 : g.a < -1e300 ? -1e300 : g.a;  // (NaN stays)
    int e = ((__double2hiint(a) >> 20) & 0x7ff) - 1023;                  // |a| < 2^(e + 1)
    if (DT == RAPID_F32 && e < 0) e = 0;
    k.a = (float)(a * __hiloint2double(::max(1023 - e, 1) << 20, 0));      // a 2^-e
    double c = (double)k.m * f.kd - g.lse2 + (double)e;
    if (DT == RAPID_BF16) c += (double)__log2f(fabsf(k.a));  // of 0: -inf
    k.c = (float)c;
    return k;
}
template <int DT>
struct Grad;
template <>
struct Grad<RAPID_BF16> {
    float k, c, nm;
    uint32_t sign;  // of a, on both halves of a pair
    __device__ __forceinline__ Grad(const GradConst& g, const Factor& f) : k(f.k), c(g.c), nm(-g.m), sign(g.a < 0.f ? 0x80008000u : 0u) {}
    __device__ __forceinline__ uint4 vector(const uint4& q) const {
        const uint32_t in[4] = {q.x, q.y, q.z, q.w};
        uint32_t out[4];
        const uint64_t k2 = f32x2(k, k), c2 = f32x2(c, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x0, x1;
            f32x2_split(f32x2_fma(bf16x2_plus(in[i], nm), k2, c2), x0, x1);
            out[i] = pack_bf16x2(ex2_approx(x0), ex2_approx(x1)) ^ sign;
        }
        return make_uint4(out[0], out[1], out[2], out[3]);
    }
    __device__ __forceinline__ uint16_t one(uint16_t z) const {
        return (uint16_t)(Elem<RAPID_BF16>::put(ex2_approx(fmaf(Elem<RAPID_BF16>::get(z) + nm, k, c))) ^ (uint16_t)sign);
    }
};
template <>
struct Grad<RAPID_F32> {
    float k, m, c, a;
    __device__ __forceinline__ Grad(const GradConst& g, const Factor& f) : k(f.k), m(g.m), c(g.c), a(g.a) {}
    __device__ __forceinline__ float one(float z) const { return a * ex2_approx(fmaf(z - m, k, c)); }
    __device__ __forceinline__ uint4 vector(const uint4& q) const {
        return make_uint4(__float_as_uint(one(__uint_as_float(q.x))), __float_as_uint(one(__uint_as_float(q.y))),
                          __float_as_uint(one(__uint_as_float(q.z))), __float_as_uint(one(__uint_as_float(q.w))));
    }
};

// Rows that count, from the preparing kernel's blocks; by one warp.
__device__ __forceinline__ long long rows_that_count(const int2* counts, int blocks) {
    long long n = 0;
    for (int i = threadIdx.x & 31; i < blocks; i += 32) n += counts[i].x;
    return warp_sum(n);
}

#endif  // __CUDACC__

// ---- what an operator brings to the rows ----------------------------------------------------------------------------

// What is made of the rows at the end: the arguments of the summing kernels, or of the last block of the rows' own kernel.
struct Totals {
    float *token, *loss;  // token may be NULL
    rapid_loss_stats_t* stats;
    int last_block;       // few rows: the rows' kernel does it
    int pieces;           // the rows' statistics are still in so many parts each (0: they are not)
};
constexpr int64_t kFewRows = 2048;
constexpr size_t kEndBytes = 2048;  // of shared memory that this takes: six sums of 32 warps, and a flag
static_assert(kEndBytes >= 32 * 6 * sizeof(double) + 1, "");

struct RowsArgs {
    const void* logits;
    void* grad;  // may be logits, may be NULL
    int64_t ld, ld_grad, n_rows;
    int vocab, dtype;
    Factor f;
    Scratch w;
    Totals end;
};

struct ClipOp {
    const int32_t* targets;
    const float *old_logp, *ref_logp, *adv;
    const int32_t* seq_rows;  // with RAPID_LOSS_NORM_SEQ
    const int2* counts;
    int count_blocks, n_seq;
    Divisor seq_len;
    uint32_t flags;
    double low, high, beta, scale, norm_z;
};
struct DistillOp {
    const int32_t* index;
    const float* logit;
    const double* teacher_lse2;
    const int2* counts;
    int64_t ld;
    int k, tail, count_blocks;
    uint32_t flags;
    double inv_tau, scale, norm_z, kd;
};

cudaError_t launch_rows(const RowsArgs& a, const ClipOp& op, int sm_count, cudaStream_t stream);
cudaError_t launch_rows(const RowsArgs& a, const DistillOp& op, int sm_count, cudaStream_t stream);

// The parts of every row's statistics and the token's logit, without a gradient; the states too, and the header.  The logits are read
// once; `keep`: they will be read again.  token_row() makes the statistics of them.
cudaError_t launch_token_stats(const RowsArgs& a, const int32_t* targets, const uint8_t* mask, bool keep, cudaStream_t stream);
// The gradient of rows whose statistics are known: coefficient coef[row / seq_len] times softmax less one at the token.
cudaError_t launch_token_grads(const RowsArgs& a, const int32_t* targets, const double* coef, const Divisor& seq_len, cudaStream_t stream);

// State of every row from mask and token, their numbers, and (where asked for) those of every generation; clears the header.
cudaError_t launch_count_by_seq(int n_seq, int seq_len, const Scratch& w, cudaStream_t stream);
cudaError_t launch_prepare_tokens(int n_seq, int seq_len, int vocab, const int32_t* targets, const uint8_t* mask, const Scratch& w,
                                  int by_seq, int* blocks, cudaStream_t stream);

#ifdef __CUDACC__


// The clipped loss of one row and its slope by the log-probability, sign turned: loss' = -slope.
struct ClipIn {
    float A, old, ref;
};
struct ClipTerms {
    double loss, slope, kl;
    bool cut;
};
__device__ __forceinline__ ClipIn clip_in(const ClipOp& op, int64_t r) {
    return ClipIn{op.adv[(op.flags & RAPID_CLIP_ADV_TOKEN) ? r : divide(r, op.seq_len)], op.old_logp[r], op.ref_logp ? op.ref_logp[r] : 0.f};
}
__device__ __forceinline__ ClipTerms clip_terms(const ClipOp& op, const ClipIn& in, double lp) {
    ClipTerms t;
    const double rho = exp2_short((lp - (double)in.old) * kLog2eD), A = (double)in.A;
    const double u = in.A != 0.f ? rho * A : 0.0;  // A = 0 leaves nothing, even of an infinite ratio
    const double v = in.A != 0.f ? fmin(fmax(rho, 1.0 - op.low), 1.0 + op.high) * A : 0.0;
    t.cut = v < u;
    t.loss = t.cut ? -v : -u;
    t.slope = t.cut ? 0.0 : u;
    t.kl = 0.0;
    if (op.ref_logp) {
        const double d = (double)in.ref - lp, e = exp2_short(d * kLog2eD) - 1.0;
        t.kl = isinf(e) ? e : e - d;  // off by 1e-15
        if (op.beta != 0.0) {
            t.loss += op.beta * t.kl;
            t.slope += op.beta * e;
        }
    }
    return t;
}
// The part of the rows' weights that all share, once for a kernel; `rows`: how many count.
__device__ __forceinline__ double shared_weight(const ClipOp& op, long long rows) {
    if (op.flags & RAPID_LOSS_NORM_GIVEN) return op.scale / op.norm_z;
    return op.scale / ((op.flags & RAPID_LOSS_NORM_SEQ) ? (double)op.n_seq : (double)rows);
}
__device__ __forceinline__ double shared_weight(const DistillOp& op, long long rows) {
    return op.scale * op.inv_tau / ((op.flags & RAPID_LOSS_NORM_GIVEN) ? op.norm_z : (double)rows);
}

// What an operator does with a row, by W lanes of a warp whose other lanes do the same for other rows.  head() reads what there is to
// read of the row in memory; look() does, ahead of time, what needs no sums over the row; finish() gives the factor once the row's
// log-sum-exp is there (without the chosen columns where exclude() says so), and is what the row's second reading waits for; values()
// gives the chosen columns' gradient and writes what is kept of the row to the scratch.  col[j] and z[j] are the chosen columns and
// their logits, t[j] the teacher's; z[j] become the columns' gradient.
__device__ __forceinline__ int list_size(const ClipOp&) { return 1; }
__device__ __forceinline__ int list_size(const DistillOp& op) { return op.k; }
__device__ __forceinline__ const int2* op_counts(const ClipOp& op) { return op.counts; }
__device__ __forceinline__ const int2* op_counts(const DistillOp& op) { return op.counts; }
__device__ __forceinline__ int op_blocks(const ClipOp& op) { return op.count_blocks; }
__device__ __forceinline__ int op_blocks(const DistillOp& op) { return op.count_blocks; }
__device__ __forceinline__ bool exclude(const ClipOp&) { return false; }
__device__ __forceinline__ bool exclude(const DistillOp& op) { return op.tail != 0; }
__device__ __forceinline__ int column(const ClipOp& op, int64_t r, int) { return op.targets[r]; }
__device__ __forceinline__ int column(const DistillOp& op, int64_t r, int j) { return op.index[r * op.ld + j]; }

__device__ __forceinline__ const float* teacher(const ClipOp&, int64_t) { return nullptr; }
__device__ __forceinline__ const float* teacher(const DistillOp& op, int64_t r) { return op.logit + r * op.ld; }

struct ClipHead {
    ClipIn in;
    int seq_rows;
};
struct ClipRow {
    ClipHead head;
    double w, lp;
};
__device__ __forceinline__ ClipHead head(const ClipOp& op, int64_t r) {
    return ClipHead{clip_in(op, r), (op.flags & RAPID_LOSS_NORM_SEQ) ? op.seq_rows[divide(r, op.seq_len)] : 1};
}
template <int W>
__device__ __forceinline__ ClipRow look(const ClipOp&, const ClipHead& in, double shared, const int*, const float*, const float*) {
    return ClipRow{in, shared, 0.0};
}
struct DistillRow {
    double teacher, w;
    double p0, lp0;   // probability of the tokens beside the list (below 0 where top_lse is too small for the list), and its logarithm
    double list_sum;  // the list's sum of 2^(x - top's x); after finish() the student's log-sum-exp over the whole vocabulary
    float top;        // the list's largest logit
};
__device__ __forceinline__ double head(const DistillOp& op, int64_t r) { return op.teacher_lse2[r]; }
template <int W>
__device__ __forceinline__ DistillRow look(const DistillOp& op, double lse2, double shared, const int* col, const float* z, const float* t) {
    const int lane = threadIdx.x % W;
    DistillRow row{lse2, shared, 0.0, 0.0, 0.0, -INFINITY};
    if (!op.tail) return row;
    double mass = 0.0;
#pragma unroll 1
    for (int j = lane; j < op.k; j += W) {
        if (col[j] < 0) continue;
        row.top = fmaxf(row.top, z[j]);
        mass += exp2_short((double)t[j] * op.kd - row.teacher);
    }
    row.top = lanes_top<W>(row.top);
    row.p0 = 1.0 - lanes_sum<W>(mass);
    if (row.p0 > 0.0) row.lp0 = log2_short(row.p0);
    if (row.top > -INFINITY)
#pragma unroll 1
        for (int j = lane; j < op.k; j += W)
            if (col[j] >= 0) row.list_sum += exp2_short(((double)z[j] - (double)row.top) * op.kd);
    row.list_sum = lanes_sum<W>(row.list_sum);
    return row;
}
__device__ __forceinline__ RowGrad finish(const ClipOp& op, const RowsArgs& a, ClipRow& row, const RowStat& st, const int*, const float* z) {
    row.lp = ((double)z[0] * a.f.kd - st.lse2) * kLn2D;
    if (op.flags & RAPID_LOSS_NORM_SEQ) row.w /= (double)row.head.seq_rows;
    return RowGrad{row.w * clip_terms(op, row.head.in, row.lp).slope, st.lse2};
}
template <int W>
__device__ __forceinline__ void values(const ClipOp&, const RowsArgs& a, int64_t r, const ClipRow& row, const RowGrad& g, const RowStat&,
                                       const int*, float* z, const float*, bool live) {
    if (threadIdx.x % W != 0 || !live) return;
    z[0] = (float)(g.a * (exp2_short(row.lp * kLog2eD) - 1.0));
    a.w.value[r] = row.lp;
}

// The teacher's probabilities together: 1, or those of the list where they come to more.  The student's term is as many times q_v.
__device__ __forceinline__ double teacher_mass(const DistillRow& row) { return row.p0 < 0.0 ? 1.0 - row.p0 : 1.0; }
// The columns outside the list: w (q_v - p_0 q_v / q_0).  Where the student has less mass there than the teacher, p_0 / q_0 is above one and
// may be beyond any type (a student that is sure of the list, or whose other columns are masked by a large negative number), while
// the gradient is not: it is then a factor w p_0 (q_0 / p_0 - 1) of the softmax over these columns alone, which st.lse2 belongs to.
__device__ __forceinline__ RowGrad finish(const DistillOp& op, const RowsArgs&, DistillRow& row, const RowStat& st, const int*, const float*) {
    RowGrad g{row.w, st.lse2};
    double& lse2 = row.list_sum;
    if (!op.tail) {
        lse2 = st.lse2;
        return g;
    }
    // the student's log-sum-exp, in a sum against the larger of the rest's and the list's largest term
    const double x0 = row.top > -INFINITY ? (double)row.top * op.kd : -INFINITY;
    const double top = fmax(st.lse2, x0);
    if (top == -INFINITY) return g;
    // (the list's sum holds its largest term, 1, so neither logarithm's argument is small)
    g.a = row.w * teacher_mass(row);
    lse2 = g.lse2 = top + log2_short(row.list_sum * exp2_short(x0 - top) + exp2_short(st.lse2 - top));
    if (row.p0 > 0.0 && st.lse2 > -INFINITY) {
        const double over = row.lp0 - (st.lse2 - lse2);  // log2 of p_0 / q_0
        const double one = 1.0 - exp2_short(-fabs(over));
        if (over > 0.0) g = RowGrad{-row.w * row.p0 * one, st.lse2};
        else g.a = row.w * one;
    }
    return g;
}
template <int W>
__device__ __forceinline__ void values(const DistillOp& op, const RowsArgs& a, int64_t r, const DistillRow& row, const RowGrad&,
                                       const RowStat& st, const int* col, float* z, const float* t, bool live) {
    const int lane = threadIdx.x % W;
    double loss = 0.0;
#pragma unroll 1
    for (int j = lane; j < op.k; j += W) {
        if (col[j] < 0) continue;
        const double lt = (double)t[j] * op.kd - row.teacher, lq = (double)z[j] * op.kd - row.list_sum;
        const double p = exp2_short(lt);
        if (p > 0.0) loss += p * (lt - lq);
        z[j] = (float)(row.w * (teacher_mass(row) * exp2_short(lq) - p));
    }
    loss = lanes_sum<W>(loss);
    if (row.p0 > 0.0) {
        // A student with nothing outside the list: infinite, unless the teacher has nothing there either.  Then p_0 is what the rounding of
        // its log-sum-exp to a float left of 0 (half a step is 2^-24 of it; four steps allow for one that was summed in float).
        const bool empty = row.p0 <= fmax(1.0, fabs(row.teacher) * kLn2D) * 0x1p-21;
        if (st.lse2 > -INFINITY || !empty) loss += row.p0 * (row.lp0 - (st.lse2 - row.list_sum));
    }
    if (lane == 0 && live) a.w.value[r] = loss * kLn2D;
}

// A row's statistics and its token's log-probability from what the reading without a gradient left of it.
__device__ __forceinline__ double token_row(const Scratch& w, int64_t r, int pieces, const Factor& f) {
    const RowStat st = stored_parts(w.parts + r * pieces, pieces);
    const double lp = ((double)w.token_z[r] * f.kd - st.lse2) * kLn2D;
    w.value[r] = lp;
    w.lse2[r] = st.lse2;
    w.row_max[r] = st.max;
    return lp;
}

// ---- sums over the rows -------------------------------------------------------------------------------------------

// Sums over the block of N numbers at once, the same in all threads; the order depends on the block's size alone.  `sh` is room for
// 32 N numbers in shared memory.
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double* sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh[warp * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? sh[lane * N + i] : 0.0);
}

// The last block of a grid to come here, with what the others wrote visible to it.  `sh` is one bool in shared memory.
__device__ __forceinline__ bool is_last_block(Header* head, bool* sh) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *sh = atomicAdd(&head->done, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (*sh) __threadfence();
    return *sh;
}

// loss, mean log-ratio, KL, rows cut, rows that count, rows that are not valid: of one row, added up
constexpr int kClipSums = 6, kDistillSums = 3;
__device__ __forceinline__ void add_row(const ClipOp& op, const Totals& t, int64_t r, const Scratch& w, const Factor& f, double (&v)[kClipSums]) {
    double lp = 0.0;
    const uint8_t st = w.state[r];
    if (st == ROW_OK) {
        lp = t.pieces ? token_row(w, r, t.pieces, f) : __ldcg(w.value + r);
        const ClipIn in = clip_in(op, r);
        const ClipTerms c = clip_terms(op, in, lp);
        v[0] += (op.flags & RAPID_LOSS_NORM_SEQ) ? c.loss / (double)op.seq_rows[divide(r, op.seq_len)] : c.loss;
        v[1] += lp - (double)in.old;
        v[2] += c.kl;
        v[3] += c.cut ? 1.0 : 0.0;
        v[4] += 1.0;
    }
    v[5] += st == ROW_BAD_TOKEN ? 1.0 : 0.0;
    if (t.token) t.token[r] = (float)lp;
}
__device__ __forceinline__ void add_row(const DistillOp&, const Totals& t, int64_t r, const Scratch& w, const Factor&, double (&v)[kDistillSums]) {
    const uint8_t st = w.state[r];
    const double l = st == ROW_OK ? __ldcg(w.value + r) : 0.0;
    v[0] += l;
    v[1] += st == ROW_OK ? 1.0 : 0.0;
    v[2] += st == ROW_BAD_TOKEN ? 1.0 : 0.0;
    if (t.token) t.token[r] = (float)l;
}
__device__ __forceinline__ void write_totals(const ClipOp& op, const Totals& t, const Scratch& w, const double (&v)[kClipSums]) {
    const long long rows = (long long)v[4];
    const double l = rows > 0 ? shared_weight(op, rows) * v[0] : 0.0, n = rows > 0 ? v[4] : 1.0;
    *t.loss = (float)l;
    if (t.stats) *t.stats = rapid_loss_stats_t{rows, (int32_t)v[3], (int32_t)v[5], 0, *(volatile int32_t*)&w.head->status, v[1] / n, v[2] / n, l};
}
__device__ __forceinline__ void write_totals(const DistillOp& op, const Totals& t, const Scratch& w, const double (&v)[kDistillSums]) {
    const long long rows = (long long)v[1];
    const double l = rows > 0 ? op.scale * v[0] / ((op.flags & RAPID_LOSS_NORM_GIVEN) ? op.norm_z : v[1]) : 0.0;
    *t.loss = (float)l;
    if (t.stats) *t.stats = rapid_loss_stats_t{rows, 0, (int32_t)v[2], 0, *(volatile int32_t*)&w.head->status, 0.0, 0.0, l};
}
template <class Op>
struct SumsOf;
template <>
struct SumsOf<ClipOp> {
    static constexpr int kN = kClipSums;
};
template <>
struct SumsOf<DistillOp> {
    static constexpr int kN = kDistillSums;
};

// By the last block of the rows' kernel, where there are few rows.  `sh`: kEndBytes of shared memory.
template <class Op>
__device__ __noinline__ void finish_rows(const Op& op, const RowsArgs& a, double* sh) {
    const Totals& t = a.end;
    const Scratch& w = a.w;
    if (!is_last_block(w.head, reinterpret_cast<bool*>(sh + 32 * SumsOf<Op>::kN))) return;
    double v[SumsOf<Op>::kN] = {};
    for (int64_t r = threadIdx.x; r < a.n_rows; r += blockDim.x) add_row(op, t, r, w, a.f, v);
    block_sums(v, sh);
    if (threadIdx.x == 0) write_totals(op, t, w, v);
}

#endif  // __CUDACC__

}  // namespace losses
}  // namespace rapid
