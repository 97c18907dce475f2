// The losses of rapid_losses.h around their rows: states and numbers of the rows before them, sums over rows, pairs and
// generations after them, and the C calls.  All of it is double and touches a few values a row, so a call's time beside the rows
// is that of the launches.
#include <algorithm>

#include "loss_rows.cuh"

namespace rapid {
namespace losses {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// ---- before the rows -------------------------------------------------------------------------------------------

__device__ __forceinline__ void clear_header(const Scratch& w) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.head = Header{0u, 0u, RAPID_OK, 0};
}

__device__ __forceinline__ void write_counts(int live, int bad, const Scratch& w) {
    __shared__ double sh[64];
    double v[2] = {(double)live, (double)bad};
    block_sums(v, sh);
    if (threadIdx.x == 0) w.counts[blockIdx.x] = make_int2((int)v[0], (int)v[1]);
}

__global__ void __launch_bounds__(kThreads)
prepare_tokens_kernel(int64_t n_rows, int vocab, const int32_t* __restrict__ targets, const uint8_t* __restrict__ mask, Scratch w) {
    clear_header(w);
    int live = 0, bad = 0;
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < n_rows; r += (int64_t)gridDim.x * kThreads) {
        uint8_t st = ROW_MASKED;
        if (!mask || mask[r]) {
            const int32_t y = targets[r];
            st = (y >= 0 && y < vocab) ? ROW_OK : ROW_BAD_TOKEN;
        }
        w.state[r] = st;
        live += st == ROW_OK;
        bad += st == ROW_BAD_TOKEN;
    }
    write_counts(live, bad, w);
}

// The same, a generation for each block, whose rows that count are noted too.
__global__ void __launch_bounds__(kThreads)
prepare_by_seq_kernel(int seq_len, int vocab, const int32_t* __restrict__ targets, const uint8_t* __restrict__ mask, Scratch w) {
    clear_header(w);
    const int64_t base = (int64_t)blockIdx.x * seq_len;
    int live = 0, bad = 0;
    for (int t = threadIdx.x; t < seq_len; t += kThreads) {
        uint8_t st = ROW_MASKED;
        if (!mask || mask[base + t]) {
            const int32_t y = targets[base + t];
            st = (y >= 0 && y < vocab) ? ROW_OK : ROW_BAD_TOKEN;
        }
        w.state[base + t] = st;
        live += st == ROW_OK;
        bad += st == ROW_BAD_TOKEN;
    }
    write_counts(live, bad, w);
    if (threadIdx.x == 0) w.seq_rows[blockIdx.x] = w.counts[blockIdx.x].x;
}

// Rows that count of every generation: one block of 32 or 256 threads each.
__global__ void __launch_bounds__(kThreads) count_by_seq_kernel(int seq_len, Scratch w) {
    const uint8_t* st = w.state + (int64_t)blockIdx.x * seq_len;
    __shared__ double sh[32];
    double n[1] = {0.0};
    for (int t = threadIdx.x; t < seq_len; t += blockDim.x) n[0] += st[t] == ROW_OK ? 1.0 : 0.0;
    block_sums(n, sh);
    if (threadIdx.x == 0) w.seq_rows[blockIdx.x] = (int)n[0];
}

// W lanes for each row, R entries a lane: whether the row's list is valid, and the teacher's log-sum-exp in base 2.
template <int W, int R>
__global__ void __launch_bounds__(kThreads)
prepare_lists_kernel(int64_t n_rows, int vocab, int k, int64_t ld, double kd, const int32_t* __restrict__ index,
                     const float* __restrict__ logit, const float* __restrict__ top_lse, const uint8_t* __restrict__ mask, Scratch w) {
    constexpr int kRows = kThreads / W;
    clear_header(w);
    const int lane = threadIdx.x % W;
    const unsigned group = W == 32 ? 0xffffffffu : ((1u << W) - 1) << (threadIdx.x & 31 & ~(W - 1));  // this row's lanes of the warp
    int live = 0, bad = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n_rows; r0 += (int64_t)gridDim.x * kRows) {  // the whole block at a time
        const int64_t r = r0 + threadIdx.x / W;
        const bool on = r < n_rows && (!mask || mask[r]);
        int v[R];
        float t[R], top = -INFINITY;
        bool some = false, wrong = false;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = W * i + lane;
            v[i] = -1 - j;  // places without an entry differ from one another
            t[i] = -INFINITY;
            if (on && j < k) {
                const int x = index[r * ld + j];
                const float z = logit[r * ld + j];
                if (x >= 0) {
                    v[i] = x;
                    t[i] = z;
                    some = true;
                    wrong |= x >= vocab || !(z < INFINITY);
                    top = fmaxf(top, z);
                }
            }
        }
        // every pair of entries once: a lane against those up to half way round, and its own
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int o = 1; o <= W / 2; ++o) wrong |= __shfl_sync(0xffffffffu, v[i], lane + o, W) == v[i];
            if (R > 1) {
#pragma unroll 4
                for (int o = 0; o < W; ++o) {
                    const int x = __shfl_sync(0xffffffffu, v[i], lane + o, W);
#pragma unroll
                    for (int i2 = i + 1; i2 < R; ++i2) wrong |= x == v[i2];
                }
            }
        }
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        some = (__ballot_sync(0xffffffffu, some) & group) != 0;
        double lse2;
        if (top_lse) {
            const float l = on ? top_lse[r] : 0.f;
            wrong |= !isfinite(l);
            lse2 = (double)l * kLog2eD;
        } else {
            some = some && top > -INFINITY;
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (t[i] > -INFINITY && t[i] < INFINITY) s += exp2_short(((double)t[i] - (double)top) * kd);
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            lse2 = s > 0.0 ? (double)top * kd + log2_short(s) : 0.0;
        }
        wrong = (__ballot_sync(0xffffffffu, wrong) & group) != 0;
        if (lane == 0 && r < n_rows) {
            const uint8_t st = !on ? ROW_MASKED : wrong ? ROW_BAD_TOKEN : some ? ROW_OK : ROW_MASKED;
            w.state[r] = st;
            w.teacher_lse2[r] = lse2;
            live += st == ROW_OK;
            bad += st == ROW_BAD_TOKEN;
        }
    }
    write_counts(live, bad, w);
}

cudaError_t launch_prepare_lists(const rapid_distill_desc_t& d, double kd, const int32_t* index, const float* logit, const float* top_lse,
                                 const uint8_t* mask, const Scratch& w, int* blocks, cudaStream_t st) {
    auto go = [&](auto kern, int width) {
        const int64_t b = (d.n_rows * width + kThreads - 1) / kThreads;
        *blocks = (int)(b < kPrepBlocks ? b : kPrepBlocks);
        kern<<<*blocks, kThreads, 0, st>>>(d.n_rows, d.vocab, d.k, d.ld_top, kd, index, logit, top_lse, mask, w);
        return cudaGetLastError();
    };
    if (d.k <= 8) return go(prepare_lists_kernel<8, 1>, 8);
    if (d.k <= 16) return go(prepare_lists_kernel<16, 1>, 16);
    if (d.k <= 32) return go(prepare_lists_kernel<32, 1>, 32);
    if (d.k <= 64) return go(prepare_lists_kernel<32, 2>, 32);
    if (d.k <= 128) return go(prepare_lists_kernel<32, 4>, 32);
    return go(prepare_lists_kernel<32, 8>, 32);
}

// ---- after the rows --------------------------------------------------------------------------------------------

// Many rows: the sums by blocks, and by the last of them over all.
template <class Op>
__global__ void __launch_bounds__(kThreads) sum_rows_kernel(Op op, Totals t, int64_t n_rows, Factor f, Scratch w) {
    constexpr int N = SumsOf<Op>::kN;
    __shared__ bool last;
    __shared__ double sh[32 * N];
    double v[N] = {};
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < n_rows; r += (int64_t)gridDim.x * kThreads) add_row(op, t, r, w, f, v);
    block_sums(v, sh);
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) w.sums[(size_t)blockIdx.x * 8 + i] = v[i];
    if (!is_last_block(w.head, &last)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0;
    for (unsigned b = threadIdx.x; b < gridDim.x; b += kThreads)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __ldcg(w.sums + (size_t)b * 8 + i);
    block_sums(v, sh);
    if (threadIdx.x == 0) write_totals(op, t, w, v);
}
template <class Op>
cudaError_t launch_sums(const Op& op, const RowsArgs& a, cudaStream_t st) {
    const int64_t b = (a.n_rows + kThreads - 1) / kThreads;
    sum_rows_kernel<<<(unsigned)(b < kSumBlocks ? b : kSumBlocks), kThreads, 0, st>>>(op, a.end, a.n_rows, a.f, a.w);
    return cudaGetLastError();
}

struct PairArgs {
    const int32_t* pairs;
    int n_pairs, n_seq, seq_len;
    uint32_t flags;
    double beta, margin, smoothing, scale, norm_z;
    float *margins, *loss;
    rapid_loss_stats_t* stats;
};
__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

// By one block: every pair's loss and slope, and their sums; returns what the slopes are multiplied by.
__device__ double pairs_of(const PairArgs& a, const Scratch& w) {
    __shared__ double sh[32 * 6];
    double v[6] = {};  // losses, margins, valid pairs, pairs won, rows, rows that are not valid
    for (int p = threadIdx.x; p < a.n_pairs; p += blockDim.x) {
        const int i = a.pairs[2 * p], j = a.pairs[2 * p + 1];
        double h = NAN, slope = 0.0;
        if (i >= 0 && i < a.n_seq && j >= 0 && j < a.n_seq) {
            h = a.beta * (__ldcg(w.seq_sum + i) - __ldcg(w.seq_sum + j)) - a.margin;
            double f;
            if (a.flags & RAPID_PREF_HINGE) {
                f = h >= 1.0 ? 0.0 : 1.0 - h;  // of NaN, NaN
                slope = h >= 1.0 ? 0.0 : h < 1.0 ? -1.0 : (double)NAN;
            } else if (a.flags & RAPID_PREF_SQUARED) {
                f = (h - 0.5) * (h - 0.5);
                slope = 2.0 * (h - 0.5);
            } else {
                f = (1.0 - a.smoothing) * softplus(-h) + (a.smoothing > 0.0 ? a.smoothing * softplus(h) : 0.0);  // (nothing times infinity)
                // e sigmoid(h) - (1 - e) sigmoid(-h), each by itself: with e = 0 a far pair's slope is small, not a difference from one
                const double t = exp(-fabs(h)), big = 1.0 / (1.0 + t), small = t * big;
                slope = h >= 0.0 ? a.smoothing * big - (1.0 - a.smoothing) * small : a.smoothing * small - (1.0 - a.smoothing) * big;
            }
            v[0] += f;
            v[1] += h;
            v[2] += 1.0;
            v[3] += h > 0.0 ? 1.0 : 0.0;
        }
        w.pair_slope[p] = slope;
        if (a.margins) a.margins[p] = (float)h;
    }
    for (int n = threadIdx.x; n < a.n_seq; n += blockDim.x) {
        v[4] += (double)__ldcg(w.seq_rows + n);
        v[5] += (double)__ldcg(w.seq_bad + n);
    }
    block_sums(v, sh);
    const double z = (a.flags & RAPID_LOSS_NORM_GIVEN) ? a.norm_z : v[2];
    if (threadIdx.x == 0) {
        const double l = v[2] > 0.0 ? a.scale * v[0] / z : 0.0, n = v[2] > 0.0 ? v[2] : 1.0;
        *a.loss = (float)l;
        if (a.stats) *a.stats = rapid_loss_stats_t{(long long)v[4], 0, (int32_t)v[5], (int32_t)v[2], RAPID_OK, v[1] / n, v[3] / n, l};
    }
    return v[2] > 0.0 ? a.scale * a.beta / z : 0.0;
}

// By one warp: minus the loss's slope by the sum of generation n's log-probabilities, over the pairs that it is in.
__device__ __forceinline__ void coefficient(const PairArgs& a, const Scratch& w, int n, double by) {
    const int lane = threadIdx.x & 31;
    double s = 0.0;
    for (int p = lane; p < a.n_pairs; p += 32) {
        const int i = a.pairs[2 * p], j = a.pairs[2 * p + 1];
        if (i == j) continue;
        if (i == n) s -= w.pair_slope[p];
        if (j == n) s += w.pair_slope[p];
    }
    s = warp_sum(s) * by;
    if (lane == 0) {
        const int rows = __ldcg(w.seq_rows + n);
        w.seq_coef[n] = (a.flags & RAPID_PREF_TOKEN_MEAN) && rows > 0 ? s / (double)rows : s;
    }
}

// One block for each generation: its sum of log-ratios.  Where there is little to do (`all`) the last one goes on to the pairs and
// the coefficients, which saves a call with few rows two launches.
__global__ void __launch_bounds__(kThreads)
pref_seq_kernel(PairArgs a, const float* __restrict__ ref_logp, float* __restrict__ token_logp, int all, int pieces, Factor f, Scratch w) {
    __shared__ bool last;
    const int64_t base = (int64_t)blockIdx.x * a.seq_len;
    __shared__ double sh[32 * 3];
    double v[3] = {};  // log-ratios, rows, rows that are not valid
    for (int t = threadIdx.x; t < a.seq_len; t += kThreads) {
        const int64_t r = base + t;
        const uint8_t st = w.state[r];
        double lp = 0.0;
        if (st == ROW_OK) {
            lp = token_row(w, r, pieces, f);
            v[0] += ref_logp ? lp - (double)ref_logp[r] : lp;
            v[1] += 1.0;
        }
        v[2] += st == ROW_BAD_TOKEN ? 1.0 : 0.0;
        if (token_logp) token_logp[r] = (float)lp;
    }
    block_sums(v, sh);
    if (threadIdx.x == 0) {
        w.seq_rows[blockIdx.x] = (int)v[1];
        w.seq_bad[blockIdx.x] = (int)v[2];
        w.seq_sum[blockIdx.x] = (a.flags & RAPID_PREF_TOKEN_MEAN) && v[1] > 0.0 ? v[0] / v[1] : v[0];
        w.seq_coef[blockIdx.x] = 0.0;  // all bits
        w.seq_top[blockIdx.x] = 0;
    }
    if (!all || !is_last_block(w.head, &last)) return;
    const double by = pairs_of(a, w);
    __syncthreads();
    for (int i = threadIdx.x >> 5; i < a.n_seq; i += kWarps) coefficient(a, w, i, by);
}

// Many pairs: every generation's slopes are added up as whole numbers, in which the order of the additions makes no difference, in two
// words: of 2^-41 of the largest of the generation's own slopes, to a power of two, and what that leaves of 2^-83 of it, so that a sum is as
// good as one in double whatever the slopes of other generations (2^20 pairs that all hold one generation come to 2^61 in either
// word at most).  A warp for each generation that goes through all pairs, as above, would be at 2^20 pairs of 2^20 generations for minutes.
constexpr int kPairThreads = 1024;
constexpr int kWordBits = 41;
constexpr double kLowWord = 4398046511104.0;  // 2^42 of the low word's are one of the high word's
__global__ void __launch_bounds__(kPairThreads) pref_pairs_kernel(PairArgs a, Scratch w) {
    const double by = pairs_of(a, w);
    if (threadIdx.x == 0) w.sums[0] = by;
}
// The largest of every generation's slopes, as the bits of a double, which for numbers of one sign are in their order (infinite ones
// and NaN above all others).  By the block above it would save a launch, and 2^20 pairs would take 3.0 ms instead of 2.0.  The sums of
// log-ratios have been read by now: their place becomes the low words'.
__global__ void __launch_bounds__(kThreads) pref_tops_kernel(PairArgs a, Scratch w) {
    const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k < a.n_seq) w.seq_sum[k] = 0.0;  // all bits
    if (k >= a.n_pairs) return;
    const int i = a.pairs[2 * k], j = a.pairs[2 * k + 1];
    const unsigned long long x = (unsigned long long)__double_as_longlong(fabs(w.pair_slope[k]));
    if (i == j || x == 0) return;  // (a pair that is left out has a slope of 0)
    if (__ldcg(w.seq_top + i) < x) atomicMax(w.seq_top + i, x);  // (what is read may be old, and is then smaller)
    if (__ldcg(w.seq_top + j) < x) atomicMax(w.seq_top + j, x);
}
__device__ __forceinline__ int top_exponent(unsigned long long top) {  // all slopes are below 2^this; of what is not finite, 1025
    return max((int)(top >> 52) - 1022, -900);
}
__device__ __forceinline__ void add_slope(const Scratch& w, int n, double x) {
    unsigned long long *high = reinterpret_cast<unsigned long long*>(w.seq_coef) + n, *low = reinterpret_cast<unsigned long long*>(w.seq_sum) + n;
    const int e = top_exponent(w.seq_top[n]);
    if (e > 1024) {  // the others make no difference; bits: one is positive, one is negative
        if (!isfinite(x)) atomicOr(high, isnan(x) ? 3ull : x > 0.0 ? 1ull : 2ull);
        return;
    }
    const double y = ldexp(x, kWordBits - e), whole = rint(y);
    atomicAdd(high, (unsigned long long)(long long)whole);
    const long long rest = (long long)rint((y - whole) * kLowWord);
    if (rest != 0) atomicAdd(low, (unsigned long long)rest);
}
__global__ void __launch_bounds__(kThreads) pref_slopes_kernel(PairArgs a, Scratch w) {
    const int p = blockIdx.x * kThreads + threadIdx.x;
    if (p >= a.n_pairs) return;
    const int i = a.pairs[2 * p], j = a.pairs[2 * p + 1];
    const double x = w.pair_slope[p];
    if (i == j || x == 0.0) return;
    add_slope(w, i, -x);
    add_slope(w, j, x);
}
__global__ void __launch_bounds__(kThreads) pref_coef_kernel(PairArgs a, Scratch w) {
    const int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (n >= a.n_seq) return;
    const int e = top_exponent(w.seq_top[n]);
    const long long high = __double_as_longlong(w.seq_coef[n]), low = __double_as_longlong(w.seq_sum[n]);
    double s;
    if (e > 1024) s = high == 3 ? (double)NAN : high == 1 ? (double)INFINITY : -(double)INFINITY;
    else s = ldexp((double)high + (double)low * (1.0 / kLowWord), e - kWordBits);
    s *= w.sums[0];
    const int rows = w.seq_rows[n];
    w.seq_coef[n] = (a.flags & RAPID_PREF_TOKEN_MEAN) && rows > 0 ? s / (double)rows : s;
}

}  // namespace

cudaError_t launch_count_by_seq(int n_seq, int seq_len, const Scratch& w, cudaStream_t stream) {
    count_by_seq_kernel<<<n_seq, seq_len > 2048 ? kThreads : 32, 0, stream>>>(seq_len, w);
    return cudaGetLastError();
}

cudaError_t launch_prepare_tokens(int n_seq, int seq_len, int vocab, const int32_t* targets, const uint8_t* mask, const Scratch& w,
                                  int by_seq, int* blocks, cudaStream_t stream) {
    if (by_seq && n_seq <= kPrepBlocks) {  // one launch instead of two
        *blocks = n_seq;
        prepare_by_seq_kernel<<<n_seq, kThreads, 0, stream>>>(seq_len, vocab, targets, mask, w);
        return cudaGetLastError();
    }
    const int64_t T = (int64_t)n_seq * seq_len, b = (T + kThreads - 1) / kThreads;
    *blocks = (int)(b < kPrepBlocks ? b : kPrepBlocks);
    prepare_tokens_kernel<<<*blocks, kThreads, 0, stream>>>(T, vocab, targets, mask, w);
    return by_seq ? launch_count_by_seq(n_seq, seq_len, w, stream) : cudaGetLastError();
}

}  // namespace losses
}  // namespace rapid

using namespace rapid;
using namespace rapid::losses;

namespace {

rapid_status_t check_scratch(const void* ws, size_t bytes, size_t need) {
    return !ws || !aligned(ws, 256) || bytes < need ? RAPID_ERR_WORKSPACE : RAPID_OK;
}
inline bool arrays_aligned(const void* a, const void* b, const void* c, const void* d, const void* e, const void* f, const void* stats) {
    return aligned(a, 4) && aligned(b, 4) && aligned(c, 4) && aligned(d, 4) && aligned(e, 4) && aligned(f, 4) && aligned(stats, 8);
}

rapid_status_t check_clip(const rapid_clip_desc_t* d) {
    if (!d || d->n_seq <= 0 || d->seq_len <= 0 || d->reserved != 0) return RAPID_ERR_INVALID_ARG;
    if (!(d->eps_low >= 0.0) || !(d->eps_high >= 0.0) || !(d->kl_beta >= 0.0) || !isfinite(d->kl_beta)) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_shape((int64_t)d->n_seq * d->seq_len, d->vocab, d->dtype, d->ld, d->ld_grad, d->flags,
                                         RAPID_LOSS_NORM_SEQ | RAPID_LOSS_NORM_GIVEN | RAPID_CLIP_ADV_TOKEN, d->scale, d->norm_z);
    // the numbers of the rows' pieces stay within 31 bits: 34 TB of logits
    return s == RAPID_OK && (int64_t)d->n_seq * d->seq_len * stat_pieces(d->vocab, d->dtype) > 0x7fffffffll ? RAPID_ERR_UNSUPPORTED : s;
}
size_t carve_clip(const rapid_clip_desc_t& d, void* base, Scratch* w) {
    return carve((int64_t)d.n_seq * d.seq_len, d.n_seq, 0, stat_pieces(d.vocab, d.dtype), (d.flags & RAPID_LOSS_NORM_SEQ) ? NEED_SEQ : 0, base, w);
}

rapid_status_t check_pref(const rapid_pref_desc_t* d) {
    if (!d || d->n_seq <= 0 || d->seq_len <= 0 || d->n_pairs <= 0) return RAPID_ERR_INVALID_ARG;
    if (!(d->beta > 0.0) || !isfinite(d->beta) || !isfinite(d->margin)) return RAPID_ERR_INVALID_ARG;
    if (!(d->label_smoothing >= 0.0 && d->label_smoothing <= 0.5)) return RAPID_ERR_INVALID_ARG;
    const uint32_t form = d->flags & (RAPID_PREF_HINGE | RAPID_PREF_SQUARED);
    if (form == (RAPID_PREF_HINGE | RAPID_PREF_SQUARED) || (form && d->label_smoothing != 0.0)) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_shape((int64_t)d->n_seq * d->seq_len, d->vocab, d->dtype, d->ld, d->ld_grad, d->flags,
                                         RAPID_LOSS_NORM_GIVEN | RAPID_PREF_HINGE | RAPID_PREF_SQUARED | RAPID_PREF_TOKEN_MEAN, d->scale,
                                         d->norm_z);
    if (s != RAPID_OK) return s;
    const int64_t pieces = std::max<int64_t>(stat_pieces(d->vocab, d->dtype), grad_pieces(d->vocab, d->dtype));
    return d->n_pairs > (1 << 20) || (int64_t)d->n_seq * d->seq_len * pieces > 0x7fffffffll ? RAPID_ERR_UNSUPPORTED : RAPID_OK;  // 17 TB
}
size_t carve_pref(const rapid_pref_desc_t& d, void* base, Scratch* w) {
    return carve((int64_t)d.n_seq * d.seq_len, d.n_seq, d.n_pairs, stat_pieces(d.vocab, d.dtype), NEED_SEQ | NEED_PAIRS, base, w);
}

rapid_status_t check_distill(const rapid_distill_desc_t* d) {
    if (!d || d->k <= 0 || d->ld_top < d->k) return RAPID_ERR_INVALID_ARG;
    if (!(d->temperature > 0.0) || !isfinite(d->temperature)) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_shape(d->n_rows, d->vocab, d->dtype, d->ld, d->ld_grad, d->flags, RAPID_LOSS_NORM_GIVEN, d->scale, d->norm_z);
    if (s != RAPID_OK) return s;
    if (d->k > kMaxList || d->ld_top > (1ll << 56) / d->n_rows) return RAPID_ERR_UNSUPPORTED;
    return d->temperature < 1e-3 || d->temperature > 1e3 ? RAPID_ERR_UNSUPPORTED : RAPID_OK;
}
size_t carve_distill(const rapid_distill_desc_t& d, void* base, Scratch* w) { return carve(d.n_rows, 0, 0, 0, NEED_TEACHER, base, w); }

inline rapid_status_t cuda_status(cudaError_t e) { return e == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA; }

}  // namespace

extern "C" {

rapid_status_t rapid_clip_loss_workspace_bytes(const rapid_clip_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_clip(desc);
    if (s == RAPID_OK) *bytes = carve_clip(*desc, nullptr, nullptr);
    return s;
}

rapid_status_t rapid_clip_loss(const rapid_clip_desc_t* desc, const void* logits, const int32_t* targets, const uint8_t* mask,
                               const float* old_logp, const float* ref_logp, const float* adv, void* dlogits, float* loss,
                               float* token_logp, rapid_loss_stats_t* stats, void* workspace, size_t workspace_bytes, void* stream) {
    rapid_status_t s = check_clip(desc);
    if (s != RAPID_OK) return s;
    const rapid_clip_desc_t& d = *desc;
    const int64_t T = (int64_t)d.n_seq * d.seq_len;
    if (!targets || !old_logp || !adv || !loss || (!ref_logp && d.kl_beta != 0.0)) return RAPID_ERR_INVALID_ARG;
    if ((s = check_matrices(logits, dlogits, T, d.vocab, d.dtype, d.ld, d.ld_grad)) != RAPID_OK) return s;
    if (!arrays_aligned(targets, old_logp, ref_logp, adv, loss, token_logp, stats)) return RAPID_ERR_ALIGNMENT;
    if ((s = check_scratch(workspace, workspace_bytes, carve_clip(d, nullptr, nullptr))) != RAPID_OK) return s;
    Scratch w;
    carve_clip(d, workspace, &w);
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool by_seq = (d.flags & RAPID_LOSS_NORM_SEQ) != 0;
    const Totals end{token_logp, loss, stats, dlogits && T <= kFewRows, dlogits ? 0 : stat_pieces(d.vocab, d.dtype)};
    const RowsArgs a{logits, dlogits, d.ld, d.ld_grad, T, d.vocab, d.dtype, make_factor(1.0, d.dtype), w, end};
    int blocks = 0;
    if (dlogits) {
        if (launch_prepare_tokens(d.n_seq, d.seq_len, d.vocab, targets, mask, w, by_seq, &blocks, st) != cudaSuccess) return RAPID_ERR_CUDA;
    } else if (launch_token_stats(a, targets, mask, false, st) != cudaSuccess || (by_seq && launch_count_by_seq(d.n_seq, d.seq_len, w, st) != cudaSuccess)) {
        return RAPID_ERR_CUDA;
    }
    const ClipOp op{targets, old_logp, ref_logp, adv, w.seq_rows, w.counts, blocks, d.n_seq, make_divisor(d.seq_len), d.flags, d.eps_low, d.eps_high,
                    d.kl_beta, d.scale, d.norm_z};
    if (dlogits && launch_rows(a, op, sms, st) != cudaSuccess) return RAPID_ERR_CUDA;
    return end.last_block ? RAPID_OK : cuda_status(launch_sums(op, a, st));
}

rapid_status_t rapid_preference_loss_workspace_bytes(const rapid_pref_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_pref(desc);
    if (s == RAPID_OK) *bytes = carve_pref(*desc, nullptr, nullptr);
    return s;
}

rapid_status_t rapid_preference_loss(const rapid_pref_desc_t* desc, const void* logits, const int32_t* targets, const uint8_t* mask,
                                     const int32_t* pairs, const float* ref_logp, void* dlogits, float* loss, float* margins,
                                     float* token_logp, rapid_loss_stats_t* stats, void* workspace, size_t workspace_bytes,
                                     void* stream) {
    rapid_status_t s = check_pref(desc);
    if (s != RAPID_OK) return s;
    const rapid_pref_desc_t& d = *desc;
    const int64_t T = (int64_t)d.n_seq * d.seq_len;
    if (!targets || !pairs || !loss) return RAPID_ERR_INVALID_ARG;
    if ((s = check_matrices(logits, dlogits, T, d.vocab, d.dtype, d.ld, d.ld_grad)) != RAPID_OK) return s;
    if (!arrays_aligned(targets, pairs, ref_logp, loss, margins, token_logp, stats)) return RAPID_ERR_ALIGNMENT;
    if ((s = check_scratch(workspace, workspace_bytes, carve_pref(d, nullptr, nullptr))) != RAPID_OK) return s;
    Scratch w;
    carve_pref(d, workspace, &w);
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RowsArgs a{logits, dlogits, d.ld, d.ld_grad, T, d.vocab, d.dtype, make_factor(1.0, d.dtype), w, Totals{}};
    if (launch_token_stats(a, targets, mask, dlogits != nullptr, st) != cudaSuccess) return RAPID_ERR_CUDA;
    const PairArgs pa{pairs, d.n_pairs, d.n_seq, d.seq_len, d.flags, d.beta, d.margin, d.label_smoothing, d.scale, d.norm_z, margins, loss, stats};
    const int all = d.n_pairs <= 4096 && (int64_t)d.n_pairs * d.n_seq <= 1 << 16;  // some ten microseconds of one block at most
    pref_seq_kernel<<<d.n_seq, kThreads, 0, st>>>(pa, ref_logp, token_logp, all, stat_pieces(d.vocab, d.dtype), a.f, w);
    if (!all) {
        pref_pairs_kernel<<<1, kPairThreads, 0, st>>>(pa, w);
        if (dlogits) {
            const unsigned by_pair = (unsigned)((d.n_pairs + kThreads - 1) / kThreads), by_seq = (unsigned)(((int64_t)d.n_seq + kThreads - 1) / kThreads);
            pref_tops_kernel<<<by_pair > by_seq ? by_pair : by_seq, kThreads, 0, st>>>(pa, w);
            pref_slopes_kernel<<<by_pair, kThreads, 0, st>>>(pa, w);
            pref_coef_kernel<<<by_seq, kThreads, 0, st>>>(pa, w);
        }
    }
    if (cudaGetLastError() != cudaSuccess) return RAPID_ERR_CUDA;
    return dlogits ? cuda_status(launch_token_grads(a, targets, w.seq_coef, make_divisor(d.seq_len), st)) : RAPID_OK;
}

rapid_status_t rapid_distill_loss_workspace_bytes(const rapid_distill_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    const rapid_status_t s = check_distill(desc);
    if (s == RAPID_OK) *bytes = carve_distill(*desc, nullptr, nullptr);
    return s;
}

rapid_status_t rapid_distill_loss(const rapid_distill_desc_t* desc, const void* logits, const int32_t* top_index, const float* top_logit,
                                  const float* top_lse, const uint8_t* mask, void* dlogits, float* loss, float* token_loss,
                                  rapid_loss_stats_t* stats, void* workspace, size_t workspace_bytes, void* stream) {
    rapid_status_t s = check_distill(desc);
    if (s != RAPID_OK) return s;
    const rapid_distill_desc_t& d = *desc;
    if (!top_index || !top_logit || !loss) return RAPID_ERR_INVALID_ARG;
    if ((s = check_matrices(logits, dlogits, d.n_rows, d.vocab, d.dtype, d.ld, d.ld_grad)) != RAPID_OK) return s;
    if (!arrays_aligned(top_index, top_logit, top_lse, loss, token_loss, nullptr, stats)) return RAPID_ERR_ALIGNMENT;
    if ((s = check_scratch(workspace, workspace_bytes, carve_distill(d, nullptr, nullptr))) != RAPID_OK) return s;
    Scratch w;
    carve_distill(d, workspace, &w);
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Factor f = make_factor(d.temperature, d.dtype);
    int blocks = 0;
    if (launch_prepare_lists(d, f.kd, top_index, top_logit, top_lse, mask, w, &blocks, st) != cudaSuccess) return RAPID_ERR_CUDA;
    const DistillOp op{top_index, top_logit, w.teacher_lse2, w.counts, d.ld_top, d.k, top_lse != nullptr, blocks, d.flags, 1.0 / d.temperature,
                       d.scale, d.norm_z, f.kd};
    const Totals end{token_loss, loss, stats, d.n_rows <= kFewRows, 0};
    const RowsArgs a{logits, dlogits, d.ld, d.ld_grad, d.n_rows, d.vocab, d.dtype, f, w, end};
    if (launch_rows(a, op, sms, st) != cudaSuccess) return RAPID_ERR_CUDA;
    return end.last_block ? RAPID_OK : cuda_status(launch_sums(op, a, st));
}

}  // extern "C"
