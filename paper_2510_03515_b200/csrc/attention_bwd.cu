// Causal attention, gradient (tcgen05).  The probabilities are recomputed from the scores and lse; nothing of size
// seq_len x seq_len touches memory, and no sum is formed by atomics, so the same inputs give the same bits.
//
// Three launches:
//   1. row terms: -delta_i = -dout_i . out_i and -lse_i in base 2, in rows padded to whole tiles; for positions without a
//      gradient the latter is -infinity, which makes their probabilities exactly zero below.
//   2. dK, dV: a block owns a key tile of one key head and walks the query tiles and the heads of the group that see it.
//          S' = K Q^T, dP' = V dO^T (rows are keys),  dV += P' dO,  dK += dS' Q     (P', dS' from tensor memory)
//   3. dQ: a block owns a query tile of one head and walks the key tiles:  S = Q K^T, dP = dO V^T, dQ += dS K.
// Scores and dP are thus formed twice: 14 instead of 10 multiply-adds a pair and element, against float atomics on dQ (or
// its partial sums in memory), which would make results depend on the order of blocks.
//
// The order of the products is such that the tensor cores have two of them to work on while the exponentials of one step are formed,
// and one or two more during its dS.
//
// Measured, 64 x 1024 positions at most, 12 heads of 128 over 2: 62 us (6.2 TB/s, the copy rate), about 205 and 190 us back to
// back, 465 in all; 545 to 610 when run for long, at 1.6 instead of 1.97 GHz under the 1000 W cap.  In a step of dK, dV of 2950 cycles the tensor cores work for
// 2048: the exponentials (1450 cycles), the product that reads them and the next scores follow one another.  Handing P' over
// in halves, or forming the next S' in halves, brought nothing (460 and 464 us against 465), nor did letting half of the row
// warps of dQ take every other step (476), or running its steps on across pieces (its kernel 211 instead of 203).
#include <math.h>

#include "attention.cuh"

namespace rapid {
namespace attn {
namespace {

// Sixteen row warps: a row's 128 columns are split over four threads, 32 columns each, so that every quarter of an SM has four
// warps whose instructions fill in for one another.  Against eight warps with 64 columns a thread (64 x 1024, 12 heads of
// 128: 218 and 238 us for the two kernels; 3 x 4095, window 1024, 16 heads of 64: 105 and 87 us) 222, 229, 99 and 77 us.
using W = Roles<16>;
constexpr int kVecBytes = kTile * 4;  // one float for each position of a tile

struct BwdArgs {
    Geometry g;
    float scale, scale_log2;
    int tiles;         // of a generation
    const float* shift;   // [n_seq][heads][tiles * 128]: -lse in base 2
    const float* ndelta;  // the same: -delta
    uint16_t *dq, *dk, *dv;
    int64_t ld_dq, ld_dk, ld_dv;
    rapid_stats_t* stats;
};

// ---- row terms --------------------------------------------------------------------------------------------------

// A block takes kTermRows positions of one generation with all their heads; 2^lanes_log2 lanes take one head of one position,
// 8 elements each, and have four of them in flight.
constexpr int kTermRows = 16;

// SHARED: generations share tiles.
template <bool SHARED>
__global__ void __launch_bounds__(256)
attn_row_terms_kernel(Geometry g, int tiles, int lanes_log2, const uint16_t* __restrict__ out, int64_t ld_out,
                      const uint16_t* __restrict__ dout, int64_t ld_dout, const float* __restrict__ lse, float* __restrict__ shift,
                      float* __restrict__ ndelta) {
    constexpr int kAhead = 4;
    const int padded = tiles * kTile, blocks = padded / kTermRows;
    const int n = (int)(blockIdx.x / (unsigned)blocks), t0 = (int)(blockIdx.x % (unsigned)blocks) * kTermRows;
    int lo, hi;
    live_range(g, n, lo, hi);
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), groups = 256 >> lanes_log2;
    const int units = kTermRows * g.heads;
    for (int u0 = 0; u0 < units; u0 += groups * kAhead) {
        const int first = u0 + (int)(threadIdx.x >> lanes_log2);
        policy::Vec8<uint16_t> x[kAhead], y[kAhead];
        int t[kAhead], h[kAhead];
        bool live[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int u = first + k * groups;
            t[k] = u / g.heads;
            h[k] = u - t[k] * g.heads;
            t[k] += t0;
            int from = lo, to = hi;
            if (SHARED) row_range(g, n, t[k], from, to);
            live[k] = u < units && t[k] >= from && t[k] < to;
            if (live[k] && lane * 8 < g.head_dim) {
                const int64_t r = (int64_t)n * g.seq_len + t[k];
                x[k].load(out + r * ld_out + h[k] * g.head_dim + lane * 8);
                y[k].load(dout + r * ld_dout + h[k] * g.head_dim + lane * 8);
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float sum = 0.f;
            if (live[k] && lane * 8 < g.head_dim) {
                float a[8], b[8];
                x[k].get(a);
                y[k].get(b);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += a[j] * b[j];
            }
            for (int o = 1; o < (1 << lanes_log2); o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0 && first + k * groups < units) {
                const int64_t at = ((int64_t)n * g.heads + h[k]) * padded + t[k];
                // double: lse * log2(e) in float would shift every score of the row by its own rounding
                shift[at] = live[k] ? (float)((double)lse[SHARED ? lse_at(g, n, h[k], t[k]) : ((size_t)n * g.heads + h[k]) * g.seq_len + t[k]] * -kLog2eD) : -INFINITY;
                ndelta[at] = -sum;
            }
        }
    }
}

// 32 scores of a row (raw, as read from tensor memory) -> exponentials of score * c + shift.  `shift_at(k)`: the pair of
// shifts of columns 2 k, 2 k + 1.
template <class F>
__device__ __forceinline__ void probabilities(const uint32_t (&s)[32], uint64_t c2, F shift_at, float (&p)[32]) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const uint64_t z = f32x2_fma(f32x2(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), c2, shift_at(k));
        float u, v;
        f32x2_split(z, u, v);
        p[2 * k] = ex2_approx(u);
        p[2 * k + 1] = ex2_approx(v);
    }
}
__device__ __forceinline__ void round_pairs(const float (&p)[32], uint32_t (&b)[16]) {
#pragma unroll
    for (int k = 0; k < 16; ++k) b[k] = pack_bf16x2(p[2 * k], p[2 * k + 1]);
}
// p * (dp - delta) as bf16
template <class F>
__device__ __forceinline__ void score_grads(const uint32_t (&s)[32], const float (&p)[32], F ndelta_at, uint32_t (&b)[16]) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        float u, v;
        f32x2_split(f32x2_mul(f32x2(p[2 * k], p[2 * k + 1]),
                              f32x2_add(f32x2(__uint_as_float(s[2 * k]), __uint_as_float(s[2 * k + 1])), ndelta_at(k))), u, v);
        b[k] = pack_bf16x2(u, v);
    }
}

// Which of a row's columns [first, first + 32) lie in [0, count): bit i for column first + i.
__device__ __forceinline__ uint32_t seen_bits(int first, unsigned count) {
    const int lo = min(max(-first, 0), 32), hi = min(max((int)count - first, 0), 32);
    const uint32_t below_hi = hi >= 32 ? 0xffffffffu : (1u << hi) - 1u, below_lo = lo >= 32 ? 0xffffffffu : (1u << lo) - 1u;
    return below_hi & ~below_lo;
}
// Columns that a row does not see <- zero, as bf16.  P and dS are masked after their rounding, each of them: in a pair that does
// not see each other the exponential or dP - delta may have overflowed, and zero times that is not zero.  (Masking the float P alone,
// whose zeros do not hold against an infinite dP: dK, dV of 64 x 1024 with 12 heads of 64 took 169 us instead of 173.)
__device__ __forceinline__ void mask_pairs(uint32_t (&b)[16], uint32_t seen) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        if (!(seen & (1u << (2 * k)))) b[k] &= 0xffff0000u;
        if (!(seen & (2u << (2 * k)))) b[k] &= 0x0000ffffu;
    }
}

// ---- dK, dV -----------------------------------------------------------------------------------------------------

// Work: a key tile of one key head; steps: the heads of its group times the query tiles that see it.
struct alignas(16) DkvWork {
    int n, hk, kt, lo, hi, q_from, q_tiles, steps;
    int end;

    __device__ __forceinline__ void set(const BwdArgs& a, int block) {
        const Geometry& g = a.g;
        end = block < 0;
        if (end) return;
        // the first key tiles are seen by the most queries: they go first
        kt = (int)((unsigned)block / (unsigned)(g.n_seq * g.kv_heads));
        const int nk = (int)((unsigned)block % (unsigned)(g.n_seq * g.kv_heads));
        n = nk / g.kv_heads;
        hk = nk - n * g.kv_heads;
        live_range(g, n, lo, hi);
        const int key_last = min(kt * kTile + kTile, hi) - 1;
        q_from = kt;
        q_tiles = 0;
        if (max(kt * kTile, lo) <= key_last) q_tiles = min(hi - 1, key_last + g.window - 1) / kTile + 1 - kt;
        steps = q_tiles * g.group;
    }
};

template <int D>
struct DkvCfg {
    static constexpr uint32_t kQ = D == 128 ? 3 : 4, kDo = D == 128 ? 2 : 4;  // tiles of q (needed the longest) and of dout in flight
    static constexpr uint32_t kVec = 2;                                       // row terms of query tiles in flight
    // At D = 128 tensor memory is full (S', dP', dV, dK): P' lies over S' and dS' over dP', each warp's part of them over its
    // own part.  At D = 64 they have columns of their own and the next S', dP' start as soon as the last are in registers.
    static constexpr bool kOverlay = D == 128;
    static constexpr size_t kTiles = (size_t)(2 + kQ + kDo) * tile_bytes<D>();
    struct Barriers {
        WorkQueue<DkvWork> queue;
        // k_*, v_*, acc_* count pieces of work that have steps, the others steps
        uint64_t k_full, v_full, acc_full, acc_empty, s_full, s_empty, dp_full, dp_empty, p_full, p_empty, ds_full, ds_empty, staged,
            all_done;
        uint64_t q_full[kQ], q_empty[kQ], q_raw[kQ], do_full[kDo], do_empty[kDo], do_raw[kDo], vec_full[kVec], vec_empty[kVec];
        uint32_t tmem_slot;
        int abort_flag;
    };
    // everything in one dynamic block, so that no byte goes to alignment: at D = 128 it fills the SM's 227 KB but for 600 bytes
    static constexpr size_t kSmem = kTiles + kVec * 2 * kVecBytes + sizeof(Barriers);
    static_assert(kSmem <= 232448, "shared memory of an SM");
};

template <int D, bool SHARED>
__global__ void __launch_bounds__(W::kThreads, 1)
attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
                const __grid_constant__ CUtensorMap mdk, const __grid_constant__ CUtensorMap mdv, const __grid_constant__ BwdArgs a) {
    using Cfg = DkvCfg<D>;
    constexpr uint32_t kQ = Cfg::kQ, kDo = Cfg::kDo, kVec = Cfg::kVec;
    constexpr bool kOverlay = Cfg::kOverlay;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ __align__(1024) uint8_t smem[];
    typename Cfg::Barriers& m = *reinterpret_cast<typename Cfg::Barriers*>(smem + Cfg::kTiles + kVec * 2 * kVecBytes);
    if ((smem_u32(smem) & 1023u) != 0) {  // the copies' swizzle counts from 1024-byte boundaries; there is no slack to move to one
        if (threadIdx.x == 0 && a.stats) atomicMax(&a.stats->status, (int)RAPID_ERR_ALIGNMENT);
        return;
    }
    volatile int* abortp = &m.abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    if (tid == 0) {
        mbar_init(&m.k_full, 1);
        mbar_init(&m.v_full, 1);
        mbar_init(&m.acc_full, 1);
        mbar_init(&m.acc_empty, W::kRow);
        mbar_init(&m.s_full, 1);
        mbar_init(&m.s_empty, W::kRow);
        mbar_init(&m.dp_full, 1);
        mbar_init(&m.dp_empty, W::kRow);
        mbar_init(&m.p_full, W::kRow);
        mbar_init(&m.p_empty, 1);
        mbar_init(&m.ds_full, W::kRow);
        mbar_init(&m.ds_empty, 1);
        mbar_init(&m.staged, W::kRow);
        mbar_init(&m.all_done, 1);
        for (uint32_t s = 0; s < kQ; ++s) {
            mbar_init(&m.q_full[s], 1);
            mbar_init(&m.q_empty[s], 1);
            mbar_init(&m.q_raw[s], 1);
        }
        for (uint32_t s = 0; s < kDo; ++s) {
            mbar_init(&m.do_full[s], 1);
            mbar_init(&m.do_empty[s], 1);
            mbar_init(&m.do_raw[s], 1);
        }
        for (uint32_t s = 0; s < kVec; ++s) {
            mbar_init(&m.vec_full[s], 1);
            mbar_init(&m.vec_empty[s], W::kRow);
        }
        work_init(&m.queue, W::kRow + 2);
        m.abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == W::kMma) {
        tmem_alloc(&m.tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, m.tmem_slot, 0);
    const uint32_t s_t = tmem, dp_t = tmem + 128u, dv_t = tmem + 256u, dk_t = tmem + 256u + D;
    const uint32_t p_t = kOverlay ? s_t : tmem + 384u, ds_t = kOverlay ? dp_t : tmem + 448u;
    constexpr uint32_t kPart = kOverlay ? 32u : 16u;  // 32-bit columns from one warp's part of P' or dS' to the next
    uint8_t* k_tile = smem;
    uint8_t* v_tile = smem + TB;
    auto q_tile = [&](uint32_t s) { return smem + (2u + s) * (uint32_t)TB; };
    auto do_tile = [&](uint32_t s) { return smem + (2u + kQ + s) * (uint32_t)TB; };
    auto vec_of = [&](uint32_t s) { return reinterpret_cast<float*>(smem + Cfg::kTiles) + s * 2u * kTile; };

    if (warp >= W::kRow) W::leave_registers();
    if (warp == W::kCopy) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0) {
            uint32_t steps = 0, n_do = 0, n_vec = 0, pieces = 0, k = 0, q_was_raw = 0, do_was_raw = 0;
            RawParity q_raw, do_raw;
            Place<kQ> qa;
            Place<kDo> da;
            Place<kVec> ca;
            bool ok = true;
            int block = (int)blockIdx.x;
            DkvWork x, last{};
            // The results of the last piece lie in its key and value tiles; they leave before new ones come.
            auto flush = [&] {
                ok = wait_one(&m.staged, (pieces - 1u) & 1u, abortp);
                if (!ok) return;
                store_tile<D>(&mdk, k_tile, g.head_dim, last.hk, last.kt * kTile, last.n);
                store_tile<D>(&mdv, v_tile, g.head_dim, last.hk, last.kt * kTile, last.n);
                bulk_commit();
                bulk_wait_read<0>();
            };
            while (true) {
                x.set(a, block);
                if (!(ok = work_put(&m.queue, k, x, abortp))) break;
                if (x.end) {
                    if (pieces > 0) flush();
                    bulk_wait_all<0>();
                    break;
                }
                int h = x.hk * g.group, qt = x.q_from;
                for (int i = 0; i < x.steps; ++i) {
                    const bool clean = dirty<SHARED>(qt, x.lo, x.hi);
                    if (steps >= kQ && !(ok = wait_one(&m.q_empty[qa.s], qa.parity ^ 1u, abortp))) break;
                    uint64_t* bar = clean ? &m.q_raw[qa.s] : &m.q_full[qa.s];
                    q_was_raw = clean ? q_was_raw | (1u << qa.s) : q_was_raw & ~(1u << qa.s);
                    if (clean) q_raw.flip(qa.s);
                    mbar_arrive_expect_tx(bar, TB);
                    load_tile<D>(q_tile(qa.s), &mq, h, qt * kTile, x.n, bar);
                    ++steps;
                    qa.step();

                    if (n_vec >= kVec && !(ok = wait_one(&m.vec_empty[ca.s], ca.parity ^ 1u, abortp))) break;
                    const size_t at = (((size_t)x.n * g.heads + h) * a.tiles + qt) * kTile;
                    mbar_arrive_expect_tx(&m.vec_full[ca.s], 2 * kVecBytes);
                    bulk_load(vec_of(ca.s), a.shift + at, kVecBytes, &m.vec_full[ca.s]);
                    bulk_load(vec_of(ca.s) + kTile, a.ndelta + at, kVecBytes, &m.vec_full[ca.s]);
                    ++n_vec;
                    ca.step();

                    if (i == 0) {
                        if (pieces > 0) flush();
                        if (!ok) break;
                        last = x;
                        mbar_arrive_expect_tx(&m.k_full, TB);
                        load_tile<D>(k_tile, &mk, x.hk, x.kt * kTile, x.n, &m.k_full);
                        mbar_arrive_expect_tx(&m.v_full, TB);
                        load_tile<D>(v_tile, &mv, x.hk, x.kt * kTile, x.n, &m.v_full);
                        ++pieces;
                    }

                    if (n_do >= kDo && !(ok = wait_one(&m.do_empty[da.s], da.parity ^ 1u, abortp))) break;
                    bar = clean ? &m.do_raw[da.s] : &m.do_full[da.s];
                    do_was_raw = clean ? do_was_raw | (1u << da.s) : do_was_raw & ~(1u << da.s);
                    if (clean) do_raw.flip(da.s);
                    mbar_arrive_expect_tx(bar, TB);
                    load_tile<D>(do_tile(da.s), &mdo, h, qt * kTile, x.n, bar);
                    ++n_do;
                    da.step();

                    if (++qt == x.q_from + x.q_tiles) {
                        qt = x.q_from;
                        ++h;
                    }
                }
                if (!ok) break;
                block = work_ask(&m.queue, k, abortp);
                if (!(ok = block >= -1)) break;
                ++k;
            }
            if (!ok || *abortp) {  // gave up: what is under way lands before the block's memory goes away
                for (uint32_t s = 0; s < kQ && s < steps; ++s) {
                    if ((q_was_raw >> s) & 1u) wait_landed(&m.q_raw[s], ((q_raw.bits >> s) & 1u) ^ 1u);
                    else wait_landed(&m.q_full[s], s < qa.s ? qa.parity : qa.parity ^ 1u);
                }
                for (uint32_t s = 0; s < kDo && s < n_do; ++s) {
                    if ((do_was_raw >> s) & 1u) wait_landed(&m.do_raw[s], ((do_raw.bits >> s) & 1u) ^ 1u);
                    else wait_landed(&m.do_full[s], s < da.s ? da.parity : da.parity ^ 1u);
                }
                for (uint32_t s = 0; s < kVec && s < n_vec; ++s) wait_landed(&m.vec_full[s], s < ca.s ? ca.parity : ca.parity ^ 1u);
                if (pieces > 0) wait_landed(&m.k_full, (pieces - 1u) & 1u);
                if (pieces > 0) wait_landed(&m.v_full, (pieces - 1u) & 1u);
            }
        }
    } else if (warp == W::kClean) {
        // ------------------------------------ dead rows ---------------------------------------------------
        RawParity q_raw, do_raw;
        Place<kQ> qa;
        Place<kDo> da;
        bool ok = true;
        DkvWork x;
        for (uint32_t k = 0; ok && work_take(&m.queue, k, x, lane, abortp); ++k) {
            int qt = x.q_from;
            for (int i = 0; i < x.steps && ok; ++i) {
                if (dirty<SHARED>(qt, x.lo, x.hi)) {
                    ok = wait_all(&m.q_raw[qa.s], q_raw.flip(qa.s), abortp);
                    if (ok) zero_dead_rows<D, SHARED>(g, q_tile(qa.s), x.n, qt * kTile, x.lo, x.hi, lane);
                    if (ok && lane == 0) mbar_arrive(&m.q_full[qa.s]);
                    ok = ok && wait_all(&m.do_raw[da.s], do_raw.flip(da.s), abortp);
                    if (ok) zero_dead_rows<D, SHARED>(g, do_tile(da.s), x.n, qt * kTile, x.lo, x.hi, lane);
                    if (ok && lane == 0) mbar_arrive(&m.do_full[da.s]);
                }
                qa.step();
                da.step();
                qt = qt + 1 < x.q_from + x.q_tiles ? qt + 1 : x.q_from;
            }
        }
    } else if (warp == W::kMma) {
        // ------------------------------------ products ----------------------------------------------------
        if (elect_one()) {
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_one(bar, parity, abortp);
                tc_fence_after();
            };
            const uint32_t kb = smem_u32(k_tile), vb = smem_u32(v_tile);
            auto q_addr = [&](uint32_t s) { return kb + (2u + s) * (uint32_t)TB; };
            auto do_addr = [&](uint32_t s) { return kb + (2u + kQ + s) * (uint32_t)TB; };
            uint32_t pieces = 0, gi = 0;   // gi: steps so far, over all pieces
            Place<kQ> qa, qd;              // the query tile of the next scores, of the next dK
            Place<kDo> da, dd;             // the dout tile of the next dP, of the next dV
            auto scores = [&] {  // S' of the next step
                wait(&m.q_full[qa.s], qa.parity);
                if (!ok) return;
                mma_rows<D>(s_t, kb, q_addr(qa.s));
                mma_commit(&m.s_full);
                qa.step();
            };
            auto dps = [&] {  // dP' of the next step
                wait(&m.do_full[da.s], da.parity);
                if (!ok) return;
                mma_rows<D>(dp_t, vb, do_addr(da.s));
                mma_commit(&m.dp_full);
                da.step();
            };
            DkvWork x;
            for (uint32_t k = 0; ok && work_take_one(&m.queue, k, x, abortp); ++k) {
                if (x.steps > 0) {
                    wait(&m.k_full, pieces & 1u);
                    if (!kOverlay && gi > 0) wait(&m.s_empty, (gi - 1u) & 1u);
                    scores();
                    wait(&m.v_full, pieces & 1u);
                    if (!kOverlay && gi > 0) wait(&m.dp_empty, (gi - 1u) & 1u);
                    dps();
                    if (pieces > 0) wait(&m.acc_empty, (pieces - 1u) & 1u);
                }
                for (int i = 0; i < x.steps && ok; ++i, ++gi) {
                    const bool more = i + 1 < x.steps;
                    if (!kOverlay && more) {
                        wait(&m.s_empty, gi & 1u);
                        scores();
                    }
                    wait(&m.p_full, gi & 1u);
                    if (!ok) break;
                    mma_sum<D>(dv_t, p_t, kPart, do_addr(dd.s), (uint32_t)i);
                    if (kOverlay && more) scores();
                    mma_commit(&m.do_empty[dd.s]);
                    dd.step();
                    if (!kOverlay) mma_commit(&m.p_empty);
                    if (!kOverlay && more) {
                        wait(&m.dp_empty, gi & 1u);
                        dps();
                    }
                    wait(&m.ds_full, gi & 1u);
                    if (!ok) break;
                    mma_sum<D>(dk_t, ds_t, kPart, q_addr(qd.s), (uint32_t)i);
                    if (!more) mma_commit(&m.acc_full);
                    if (kOverlay && more) dps();
                    mma_commit(&m.q_empty[qd.s]);
                    qd.step();
                    if (!kOverlay) mma_commit(&m.ds_empty);
                }
                if (x.steps > 0) ++pieces;
            }
            // every product has ended before tensor memory is given back
            mma_commit(&m.all_done);
            wait_drained(&m.all_done, abortp);
        }
        __syncwarp();
    } else if (warp < W::kRow) {
        // ------------------------------------ probabilities, dS -------------------------------------------
        W::take_registers();
        const int part = warp >> 2, row = (warp & 3) * 32 + lane;  // columns [32 part, 32 part + 32)
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mine = lanes + (uint32_t)part * 32u, packed = lanes + (uint32_t)part * kPart;
        const uint64_t c2 = f32x2(a.scale_log2, a.scale_log2);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && wait_all(bar, parity, abortp);
            tc_fence_after();
            return ok;
        };
        auto tell = [&](uint64_t* bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        uint32_t gi = 0, pieces = 0;
        Place<kVec> ca;
        DkvWork x;
        for (uint32_t k = 0; work_take(&m.queue, k, x, lane, abortp); ++k) {
            const int key = x.kt * kTile + row;
            int lo = x.lo, hi = x.hi;
            if (SHARED) row_range(g, x.n, key, lo, hi);
            const unsigned seen_by = !SHARED ? (unsigned)g.window : (unsigned)max(0, min(g.window, hi - key));  // queries from `key` on
            int qt = x.q_from;
            for (int i = 0; i < x.steps; ++i, ++gi) {
                const int q0 = qt * kTile;
                qt = qt + 1 < x.q_from + x.q_tiles ? qt + 1 : x.q_from;
                float p[32];
                uint32_t s[32], b[16];
                if (!wait(&m.vec_full[ca.s], ca.parity) || !wait(&m.s_full, gi & 1u)) break;
                tmem_ld32(s_t + mine, s);
                tmem_ld_wait();
                if (!kOverlay) tell(&m.s_empty);
                const ulonglong2* shift = reinterpret_cast<const ulonglong2*>(vec_of(ca.s) + part * 32);
                probabilities(s, c2, [&](int e) { return e & 1 ? shift[e >> 1].y : shift[e >> 1].x; }, p);
                // the diagonal, and the far edge of a window
                const uint32_t seen = seen_bits(q0 + part * 32 - key, seen_by);
                // a warp whose rows see all of its columns has nothing to mask
                const bool edge = (q0 <= x.kt * kTile || q0 + kTile - 1 - x.kt * kTile >= g.window) && !__all_sync(0xffffffffu, seen == 0xffffffffu);
                round_pairs(p, b);
                if (edge) mask_pairs(b, seen);
                if (!kOverlay && gi > 0 && !wait(&m.p_empty, (gi - 1u) & 1u)) break;
                tmem_st16(p_t + packed, b);
                tmem_st_wait();
                tell(&m.p_full);

                if (!wait(&m.dp_full, gi & 1u)) break;
                tmem_ld32(dp_t + mine, s);
                tmem_ld_wait();
                if (!kOverlay) tell(&m.dp_empty);
                const ulonglong2* ndelta = reinterpret_cast<const ulonglong2*>(vec_of(ca.s) + kTile + part * 32);
                score_grads(s, p, [&](int e) { return e & 1 ? ndelta[e >> 1].y : ndelta[e >> 1].x; }, b);
                if (edge) mask_pairs(b, seen);
                if (!kOverlay && gi > 0 && !wait(&m.ds_empty, (gi - 1u) & 1u)) break;
                tmem_st16(ds_t + packed, b);
                tmem_st_wait();
                tell(&m.ds_full);
                if (lane == 0) mbar_arrive(&m.vec_empty[ca.s]);
                ca.step();
            }
            // half of the warps write dV, half dK, each half of the columns
            if (ok && x.steps > 0) wait(&m.acc_full, pieces & 1u);
            if (!ok) break;
            const bool keys = part >= 2;
            if (x.steps > 0) {
                const bool live = key >= lo && key < hi;
#pragma unroll 1
                for (int c = (part & 1) * (D / 64); c < ((part & 1) + 1) * (D / 64); ++c)
                    stage_acc32(keys ? k_tile : v_tile, row, c, (keys ? dk_t : dv_t) + lanes + 32u * c, live, keys ? a.scale : 1.f);
                fence_proxy_async_smem();
                tell(&m.acc_empty);
                tell(&m.staged);
                ++pieces;
            } else {
                zero_tile(keys ? a.dk : a.dv, keys ? a.ld_dk : a.ld_dv, g.seq_len, g.head_dim, x.hk, x.kt * kTile, x.n,
                          (part & 1) * 128 + row, 256);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == W::kMma) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && m.abort_flag && a.stats) atomicMax(&a.stats->status, (int)RAPID_ERR_TIMEOUT);
}

// ---- dQ ---------------------------------------------------------------------------------------------------------

template <int D>
struct DqCfg {
    static constexpr int kKeys = D == 128 ? 3 : 4, kVals = D == 128 ? 2 : 3;  // tiles of keys (needed for two steps) and values in flight
    static constexpr size_t kSmem = (size_t)(2 + kKeys + kVals) * tile_bytes<D>() + 1024;
};

// Work: a query tile of one head; steps: the key tiles that it sees.
struct alignas(16) DqWork {
    int n, h, t, lo, hi, from, steps;
    int end;

    __device__ __forceinline__ void set(const BwdArgs& a, int block) {
        const Geometry& g = a.g;
        end = block < 0;
        if (end) return;
        // the longest rows first; the heads of a group next to one another, they read the same keys
        t = a.tiles - 1 - (int)((unsigned)block / (unsigned)(g.n_seq * g.heads));
        const int nh = (int)((unsigned)block % (unsigned)(g.n_seq * g.heads));
        n = nh / g.heads;
        h = nh - n * g.heads;
        live_range(g, n, lo, hi);
        int to;
        key_tiles(g, t, lo, hi, from, to);
        steps = to - from;
    }
};

template <int D, bool SHARED>
__global__ void __launch_bounds__(W::kThreads, 1)
attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
               const __grid_constant__ CUtensorMap mdq, const __grid_constant__ BwdArgs a) {
    constexpr uint32_t kKeys = DqCfg<D>::kKeys, kVals = DqCfg<D>::kVals;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // q_*, do_*, acc_* count pieces of work that have steps, the others steps
    __shared__ __align__(8) uint64_t q_full, q_empty, do_full, do_empty, acc_full, acc_empty, s_full[2], dp_full, ds_full, all_done, staged[kKeys],
        k_full[kKeys], k_empty[kKeys], k_raw[kKeys], v_full[kVals], v_empty[kVals], v_raw[kVals];
    __shared__ __align__(16) WorkQueue<DqWork> queue;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* abortp = &abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    if (tid == 0) {
        mbar_init(&q_full, 1);
        mbar_init(&q_empty, 1);
        mbar_init(&do_full, 1);
        mbar_init(&do_empty, 1);
        mbar_init(&acc_full, 1);
        mbar_init(&acc_empty, W::kRow);
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        mbar_init(&dp_full, 1);
        mbar_init(&ds_full, W::kRow);
        mbar_init(&all_done, 1);
        for (uint32_t s = 0; s < kKeys; ++s) {
            mbar_init(&k_full[s], 1);
            mbar_init(&k_empty[s], 1);
            mbar_init(&k_raw[s], 1);
            mbar_init(&staged[s], W::kRow);
        }
        for (uint32_t s = 0; s < kVals; ++s) {
            mbar_init(&v_full[s], 1);
            mbar_init(&v_empty[s], 1);
            mbar_init(&v_raw[s], 1);
        }
        work_init(&queue, W::kRow + 2);
        abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == W::kMma) {
        tmem_alloc(&tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    // scores of even and odd steps (dS of a step lies over its scores), dP, dQ
    auto s_addr = [&](uint32_t i) { return tmem + (i & 1u) * 128u; };
    const uint32_t dp_t = tmem + 256u, dq_t = tmem + 384u;
    uint8_t* q_tile = smem;
    uint8_t* do_tile = smem + TB;
    auto k_tile = [&](uint32_t s) { return smem + (2u + s) * (uint32_t)TB; };
    auto v_tile = [&](uint32_t s) { return smem + (2u + kKeys + s) * (uint32_t)TB; };

    if (warp >= W::kRow) W::leave_registers();
    if (warp == W::kCopy) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0) {
            bool ok = true;
            uint32_t nk = 0, nv = 0, nq = 0, ndo = 0, k = 0, k_was_raw = 0, v_was_raw = 0;
            RawParity kr, vr;
            Place<kKeys> ka;
            Place<kVals> va;
            int block = (int)blockIdx.x;
            DqWork x;
            // The results of a piece are left in the place of its last key tile, the buffer that is wanted again last: they
            // leave when a new tile is to go there, or at the end.
            RawParity staged_at;
            uint32_t pending = 0;  // buffers that hold results
            int held[kKeys][3];    // whose
            auto flush = [&](uint32_t s) {
                if (!((pending >> s) & 1u)) return;
                pending &= ~(1u << s);
                ok = wait_one(&staged[s], staged_at.flip(s), abortp);
                if (!ok) return;
                int h = 0, t = 0, n = 0;
#pragma unroll
                for (uint32_t i = 0; i < kKeys; ++i)
                    if (i == s) h = held[i][0], t = held[i][1], n = held[i][2];
                store_tile<D>(&mdq, k_tile(s), g.head_dim, h, t * kTile, n);
                bulk_commit();
                bulk_wait_read<0>();
            };
            while (true) {
                x.set(a, block);
                if (!(ok = work_put(&queue, k, x, abortp))) break;
                if (x.end) {
                    for (uint32_t i = 0; i < kKeys && ok; ++i, ka.step()) flush(ka.s);  // the oldest first
                    bulk_wait_all<0>();
                    break;
                }
                if (x.steps > 0) {
                    if (nq > 0 && !(ok = wait_one(&q_empty, (nq - 1u) & 1u, abortp))) break;
                    mbar_arrive_expect_tx(&q_full, TB);
                    load_tile<D>(q_tile, &mq, x.h, x.t * kTile, x.n, &q_full);
                    ++nq;
                }
                // in the order of use: K_0 dout V_0 K_1 V_1 ...
                const int hk = x.h / g.group;
                for (int i = 0; i < x.steps; ++i) {
                    const int t0 = (x.from + i) * kTile;
                    const bool clean = dirty<SHARED>(x.from + i, x.lo, x.hi);
                    if (nk >= kKeys && !(ok = wait_one(&k_empty[ka.s], ka.parity ^ 1u, abortp))) break;
                    flush(ka.s);
                    if (!ok) break;
                    if (i + 1 == x.steps) {
                        pending |= 1u << ka.s;
#pragma unroll
                        for (uint32_t b = 0; b < kKeys; ++b)
                            if (b == ka.s) held[b][0] = x.h, held[b][1] = x.t, held[b][2] = x.n;
                    }
                    uint64_t* bar = clean ? &k_raw[ka.s] : &k_full[ka.s];
                    k_was_raw = clean ? k_was_raw | (1u << ka.s) : k_was_raw & ~(1u << ka.s);
                    if (clean) kr.flip(ka.s);
                    mbar_arrive_expect_tx(bar, TB);
                    load_tile<D>(k_tile(ka.s), &mk, hk, t0, x.n, bar);
                    ++nk;
                    ka.step();
                    if (i == 0) {
                        if (ndo > 0 && !(ok = wait_one(&do_empty, (ndo - 1u) & 1u, abortp))) break;
                        mbar_arrive_expect_tx(&do_full, TB);
                        load_tile<D>(do_tile, &mdo, x.h, x.t * kTile, x.n, &do_full);
                        ++ndo;
                    }
                    if (nv >= kVals && !(ok = wait_one(&v_empty[va.s], va.parity ^ 1u, abortp))) break;
                    bar = clean ? &v_raw[va.s] : &v_full[va.s];
                    v_was_raw = clean ? v_was_raw | (1u << va.s) : v_was_raw & ~(1u << va.s);
                    if (clean) vr.flip(va.s);
                    mbar_arrive_expect_tx(bar, TB);
                    load_tile<D>(v_tile(va.s), &mv, hk, t0, x.n, bar);
                    ++nv;
                    va.step();
                }
                if (!ok) break;
                block = work_ask(&queue, k, abortp);
                if (!(ok = block >= -1)) break;
                ++k;
            }
            if (!ok || *abortp) {  // gave up: what is under way lands before the block's memory goes away
                if (nq > 0) wait_landed(&q_full, (nq - 1u) & 1u);
                if (ndo > 0) wait_landed(&do_full, (ndo - 1u) & 1u);
                for (uint32_t s = 0; s < kKeys && s < nk; ++s) {
                    if ((k_was_raw >> s) & 1u) wait_landed(&k_raw[s], ((kr.bits >> s) & 1u) ^ 1u);
                    else wait_landed(&k_full[s], s < ka.s ? ka.parity : ka.parity ^ 1u);
                }
                for (uint32_t s = 0; s < kVals && s < nv; ++s) {
                    if ((v_was_raw >> s) & 1u) wait_landed(&v_raw[s], ((vr.bits >> s) & 1u) ^ 1u);
                    else wait_landed(&v_full[s], s < va.s ? va.parity : va.parity ^ 1u);
                }
            }
        }
    } else if (warp == W::kClean) {
        // ------------------------------------ dead rows ---------------------------------------------------
        RawParity kr, vr;
        Place<kKeys> ka;
        Place<kVals> va;
        bool ok = true;
        DqWork x;
        for (uint32_t k = 0; ok && work_take(&queue, k, x, lane, abortp); ++k) {
            for (int i = 0; i < x.steps && ok; ++i) {
                const int t0 = (x.from + i) * kTile;
                if (dirty<SHARED>(x.from + i, x.lo, x.hi)) {
                    ok = wait_all(&k_raw[ka.s], kr.flip(ka.s), abortp);
                    if (ok) zero_dead_rows<D, SHARED>(g, k_tile(ka.s), x.n, t0, x.lo, x.hi, lane);
                    if (ok && lane == 0) mbar_arrive(&k_full[ka.s]);
                    ok = ok && wait_all(&v_raw[va.s], vr.flip(va.s), abortp);
                    if (ok) zero_dead_rows<D, SHARED>(g, v_tile(va.s), x.n, t0, x.lo, x.hi, lane);
                    if (ok && lane == 0) mbar_arrive(&v_full[va.s]);
                }
                ka.step();
                va.step();
            }
        }
    } else if (warp == W::kMma) {
        // ------------------------------------ products ----------------------------------------------------
        if (elect_one()) {
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = ok && wait_one(bar, parity, abortp);
                tc_fence_after();
            };
            const uint32_t qb = smem_u32(q_tile), dob = smem_u32(do_tile);
            auto k_addr = [&](uint32_t s) { return qb + (2u + s) * (uint32_t)TB; };
            auto v_addr = [&](uint32_t s) { return qb + (2u + kKeys + s) * (uint32_t)TB; };
            uint32_t pieces = 0, gi = 0, gs = 0;  // gi: steps so far; gs: scores so far
            Place<kKeys> ka, kd;                  // the key tile of the next scores, of the next dQ
            Place<kVals> va;
            auto scores = [&](bool last) {
                wait(&k_full[ka.s], ka.parity);
                if (!ok) return;
                mma_rows<D>(s_addr(gs), qb, k_addr(ka.s));
                mma_commit(&s_full[gs & 1u]);
                if (last) mma_commit(&q_empty);
                ka.step();
                ++gs;
            };
            auto dps = [&](bool last) {
                if (!ok) return;
                mma_rows<D>(dp_t, dob, v_addr(va.s));
                mma_commit(&dp_full);
                mma_commit(&v_empty[va.s]);
                if (last) mma_commit(&do_empty);
                va.step();
            };
            DqWork x;
            for (uint32_t k = 0; ok && work_take_one(&queue, k, x, abortp); ++k) {
                if (x.steps > 0) {
                    wait(&q_full, pieces & 1u);
                    scores(x.steps == 1);
                    wait(&do_full, pieces & 1u);
                    wait(&v_full[va.s], va.parity);
                    dps(x.steps == 1);
                    if (x.steps > 1) scores(x.steps == 2);
                    if (pieces > 0) wait(&acc_empty, (pieces - 1u) & 1u);
                }
                for (int i = 0; i < x.steps && ok; ++i, ++gi) {
                    if (i + 1 < x.steps) wait(&v_full[va.s], va.parity);
                    wait(&ds_full, gi & 1u);  // dP has been read, dS is there
                    if (i + 1 < x.steps) dps(i + 2 == x.steps);
                    if (!ok) break;
                    mma_sum<D>(dq_t, s_addr(gi), 32u, k_addr(kd.s), (uint32_t)i);
                    if (i + 1 == x.steps) mma_commit(&acc_full);
                    mma_commit(&k_empty[kd.s]);
                    kd.step();
                    if (i + 2 < x.steps) scores(i + 3 == x.steps);
                }
                if (x.steps > 0) ++pieces;
            }
            mma_commit(&all_done);
            wait_drained(&all_done, abortp);
        }
        __syncwarp();
    } else if (warp < W::kRow) {
        // ------------------------------------ probabilities, dS -------------------------------------------
        W::take_registers();
        const int part = warp >> 2, row = (warp & 3) * 32 + lane;  // columns [32 part, 32 part + 32)
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mine = lanes + (uint32_t)part * 32u;
        const uint64_t c2 = f32x2(a.scale_log2, a.scale_log2);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && wait_all(bar, parity, abortp);
            tc_fence_after();
            return ok;
        };
        auto tell = [&](uint64_t* bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        uint32_t gi = 0, pieces = 0;
        Place<kKeys> kc;  // the key tile of this step
        uint32_t key_buf = 0;
        // A piece and its row's terms; the next one is taken, and its terms are asked for, before this one's dQ is waited for.
        DqWork x;
        float shift = 0.f, ndelta = 0.f;
        auto take = [&](uint32_t k) {
            if (!work_take(&queue, k, x, lane, abortp)) return false;
            const size_t at = (((size_t)x.n * g.heads + x.h) * a.tiles + x.t) * kTile + row;
            shift = a.shift[at];
            ndelta = a.ndelta[at];
            return true;
        };
        bool more = take(0);
        for (uint32_t k = 1; more; ++k) {
            const int pos = x.t * kTile + row;
            int lo = x.lo, hi = x.hi;
            if (SHARED) row_range(g, x.n, pos, lo, hi);
            const bool live = pos >= lo && pos < hi;
            const int see = max(lo, pos - g.window + 1);
            const unsigned count = live ? (unsigned)(pos + 1 - see) : 0u;
            int full_from = 1 << 30, full_to = 0;  // key tiles that every row of the tile sees whole
            if (!SHARED && x.t * kTile >= x.lo && x.t * kTile + kTile <= x.hi) {
                full_from = (max(x.lo, x.t * kTile + kTile - g.window) + kTile - 1) / kTile;
                full_to = x.t;
            }
            const uint64_t shift2 = f32x2(shift, shift), ndelta2 = f32x2(ndelta, ndelta);
            for (int i = 0; i < x.steps; ++i, ++gi) {
                const int j = x.from + i;
                key_buf = kc.s;
                kc.step();
                float p[32];
                uint32_t s[32], b[16];
                if (!wait(&s_full[gi & 1u], (gi >> 1) & 1u)) break;
                tmem_ld32(s_addr(gi) + mine, s);
                tmem_ld_wait();
                probabilities(s, c2, [&](int) { return shift2; }, p);
                const uint32_t seen = seen_bits(j * kTile + part * 32 - see, count);
                const bool edge = (j < full_from || j >= full_to) && !__all_sync(0xffffffffu, seen == 0xffffffffu);
                if (!wait(&dp_full, gi & 1u)) break;
                tmem_ld32(dp_t + mine, s);
                tmem_ld_wait();
                score_grads(s, p, [&](int) { return ndelta2; }, b);
                if (edge) mask_pairs(b, seen);
                tmem_st16(s_addr(gi) + mine, b);
                tmem_st_wait();
                tell(&ds_full);
            }
            const int n = x.n, h = x.h, t = x.t;
            const bool any = x.steps > 0;
            if (!ok) break;
            more = take(k);
            if (any && !wait(&acc_full, pieces & 1u)) break;
            if (any) {  // 32 columns each (at D = 64 half of the warps have none)
                if (part * 32 < D) stage_acc32(k_tile(key_buf), row, part, dq_t + lanes + 32u * part, live, a.scale);
                fence_proxy_async_smem();
                tell(&acc_empty);
                tell(&staged[key_buf]);
                ++pieces;
            } else {
                zero_tile(a.dq, a.ld_dq, g.seq_len, g.head_dim, h, t * kTile, n, part * 128 + row, 512);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == W::kMma) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && abort_flag && a.stats) atomicMax(&a.stats->status, (int)RAPID_ERR_TIMEOUT);
}

// ---- host -------------------------------------------------------------------------------------------------------

struct Maps {
    CUtensorMap q, k, v, dout, dq, dk, dv;
};

template <int D, bool SHARED>
cudaError_t launch_bwd(const Maps& m, const BwdArgs& a, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(attn_dkv_kernel<D, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DkvCfg<D>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_dq_kernel<D, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DqCfg<D>::kSmem);
    if (e != cudaSuccess) return e;
    const unsigned nk = (unsigned)(a.g.n_seq * a.g.kv_heads), nh = (unsigned)(a.g.n_seq * a.g.heads);
    attn_dkv_kernel<D, SHARED><<<nk * (unsigned)a.tiles, W::kThreads, DkvCfg<D>::kSmem, st>>>(m.q, m.k, m.v, m.dout, m.dk, m.dv, a);
    attn_dq_kernel<D, SHARED><<<nh * (unsigned)a.tiles, W::kThreads, DqCfg<D>::kSmem, st>>>(m.q, m.k, m.v, m.dout, m.dq, a);
    return cudaGetLastError();
}

rapid_status_t check_attn_bwd(const rapid_attn_desc_t* d) {
    rapid_status_t s = check_attn(d);
    if (s != RAPID_OK) return s;
    const int64_t wq = (int64_t)d->n_heads * d->head_dim, wk = (int64_t)d->n_kv_heads * d->head_dim;
    if (d->ld_dout < wq || d->ld_dq < wq || d->ld_dk < wk || d->ld_dv < wk) return RAPID_ERR_INVALID_ARG;
    if (d->ld_dout % 8 || d->ld_dq % 8 || d->ld_dk % 8 || d->ld_dv % 8) return RAPID_ERR_ALIGNMENT;
    const int64_t most = (1ll << 38) / d->seq_len < (1ll << 31) ? (1ll << 38) / d->seq_len : (1ll << 31);
    if (d->ld_dout > most || d->ld_dq > most || d->ld_dk > most || d->ld_dv > most) return RAPID_ERR_UNSUPPORTED;
    // A piece of dK, dV is one key tile's walk over the query tiles that see it, for all heads of its group.  A warp that has no dead
    // rows to clear in it waits for the next piece meanwhile; 2^20 steps of 1.5 us (2.3 at 1.3 GHz) stay below that wait's limit.
    const int64_t tiles = (d->seq_len + kTile - 1) / kTile, in_window = d->window ? ((int64_t)d->window + kTile - 2) / kTile + 1 : tiles;
    if ((in_window < tiles ? in_window : tiles) * (d->n_heads / d->n_kv_heads) > (1 << 20)) return RAPID_ERR_UNSUPPORTED;
    return RAPID_OK;
}

// Floats of one of the two arrays: what the larger share needs (they follow one another), in whole 8 KB.
size_t row_terms(const rapid_attn_desc_t& d) {
    Share shares[2];
    const int count = make_shares(d, nullptr, shares);
    size_t most = 0;
    for (int i = 0; i < count; ++i) {
        const rapid_attn_desc_t& s = shares[i].d;
        const size_t floats = (size_t)((s.seq_len + kTile - 1) / kTile) * kTile * (size_t)s.n_seq * (size_t)s.n_heads;
        most = floats > most ? floats : most;
    }
    return align_up(most, 2048);
}

}  // namespace
}  // namespace attn
}  // namespace rapid

using namespace rapid;
using namespace rapid::attn;

extern "C" rapid_status_t rapid_attention_bwd_workspace_bytes(const rapid_attn_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    rapid_status_t s = check_attn_bwd(desc);
    if (s != RAPID_OK) return s;
    *bytes = row_terms(*desc) * 2 * sizeof(float);
    return RAPID_OK;
}

extern "C" rapid_status_t rapid_attention_bwd(const rapid_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                              const int32_t* bounds, const void* out, const float* lse, const void* dout, void* dq,
                                              void* dk, void* dv, rapid_stats_t* stats, void* workspace, size_t workspace_bytes,
                                              void* stream) {
    rapid_status_t s = check_attn_bwd(desc);
    if (s != RAPID_OK) return s;
    const rapid_attn_desc_t& d = *desc;
    const void* in[5] = {q, k, v, out, dout};
    void* grads[3] = {dq, dk, dv};
    if (!lse) return RAPID_ERR_INVALID_ARG;
    for (const void* p : in)
        if (!p) return RAPID_ERR_INVALID_ARG;
    for (const void* p : grads)
        if (!p) return RAPID_ERR_INVALID_ARG;
    for (const void* p : in)
        if (!policy::aligned(p, 16)) return RAPID_ERR_ALIGNMENT;
    for (const void* p : grads)
        if (!policy::aligned(p, 16)) return RAPID_ERR_ALIGNMENT;
    if (!policy::aligned(bounds, 4) || !policy::aligned(lse, 4) || !policy::aligned(stats, 8)) return RAPID_ERR_ALIGNMENT;
    const int64_t T = (int64_t)d.n_seq * d.seq_len, wq = (int64_t)d.n_heads * d.head_dim, wk = (int64_t)d.n_kv_heads * d.head_dim;
    const int64_t in_w[5] = {wq, wk, wk, wq, wq}, in_ld[5] = {d.ld_q, d.ld_k, d.ld_v, d.ld_out, d.ld_dout};
    const int64_t g_w[3] = {wq, wk, wk}, g_ld[3] = {d.ld_dq, d.ld_dk, d.ld_dv};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 5; ++j)
            if (policy::rows_overlap(grads[i], g_w[i], g_ld[i], in[j], in_w[j], in_ld[j], T, 2)) return RAPID_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (policy::rows_overlap(grads[i], g_w[i], g_ld[i], grads[j], g_w[j], g_ld[j], T, 2)) return RAPID_ERR_INVALID_ARG;
    }
    const size_t terms = row_terms(d);
    if (!workspace || !policy::aligned(workspace, 256) || workspace_bytes < terms * 2 * sizeof(float)) return RAPID_ERR_WORKSPACE;
    int sms = 0;
    if ((s = policy::check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (policy::clear_stats(stats, st) != cudaSuccess) return RAPID_ERR_CUDA;
    int lanes_log2 = 0;
    while ((8 << lanes_log2) < d.head_dim) ++lanes_log2;
    Share shares[2];
    const int count = make_shares(d, bounds, shares);
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < count && e == cudaSuccess; ++i) {
        const Share& c = shares[i];
        const void *o_rows = rows_from(out, c.first_row, d.ld_out), *do_rows = rows_from(dout, c.first_row, d.ld_dout);
        void *dq_rows = rows_from(dq, c.first_row, d.ld_dq), *dk_rows = rows_from(dk, c.first_row, d.ld_dk),
             *dv_rows = rows_from(dv, c.first_row, d.ld_dv);
        Maps m;
        if (!make_head_map(&m.q, rows_from(q, c.first_row, d.ld_q), c.d, d.n_heads, d.ld_q) ||
            !make_head_map(&m.k, rows_from(k, c.first_row, d.ld_k), c.d, d.n_kv_heads, d.ld_k) ||
            !make_head_map(&m.v, rows_from(v, c.first_row, d.ld_v), c.d, d.n_kv_heads, d.ld_v) ||
            !make_head_map(&m.dout, do_rows, c.d, d.n_heads, d.ld_dout) || !make_head_map(&m.dq, dq_rows, c.d, d.n_heads, d.ld_dq) ||
            !make_head_map(&m.dk, dk_rows, c.d, d.n_kv_heads, d.ld_dk) || !make_head_map(&m.dv, dv_rows, c.d, d.n_kv_heads, d.ld_dv))
            return RAPID_ERR_CUDA;
        BwdArgs a;
        a.g = c.g;
        a.scale = (float)d.scale;
        a.scale_log2 = (float)(d.scale * kLog2eD);
        a.tiles = (c.d.seq_len + kTile - 1) / kTile;
        // the second share's row terms take the place of the first's, which its kernels have read by then
        a.shift = static_cast<float*>(workspace);
        float* ndelta = static_cast<float*>(workspace) + terms;
        a.ndelta = ndelta;
        a.dq = static_cast<uint16_t*>(dq_rows);
        a.dk = static_cast<uint16_t*>(dk_rows);
        a.dv = static_cast<uint16_t*>(dv_rows);
        a.ld_dq = d.ld_dq;
        a.ld_dk = d.ld_dk;
        a.ld_dv = d.ld_dv;
        a.stats = stats;
        const int64_t blocks = (int64_t)c.d.n_seq * a.tiles * (kTile / kTermRows);
        if (blocks > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;
        auto terms_kernel = c.g.part ? attn_row_terms_kernel<true> : attn_row_terms_kernel<false>;
        terms_kernel<<<(unsigned)blocks, 256, 0, st>>>(a.g, a.tiles, lanes_log2, static_cast<const uint16_t*>(o_rows), d.ld_out,
                                                       static_cast<const uint16_t*>(do_rows), d.ld_dout, lse + c.first_row * d.n_heads,
                                                       static_cast<float*>(workspace), ndelta);
        auto launch = d.head_dim <= 64 ? (c.g.part ? launch_bwd<64, true> : launch_bwd<64, false>)
                                       : (c.g.part ? launch_bwd<128, true> : launch_bwd<128, false>);
        e = launch(m, a, st);
    }
    return e == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
