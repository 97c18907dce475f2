// Causal attention, forward (tcgen05).
//
// A piece of work is two items of one key head: an item is (query tile of 128 positions, query head of the group), items
// are numbered tile by tile, so the two usually share the tile and always the keys.  Four warps run the softmax of one item, a
// thread to a row, so row maximum and sum need no exchange:
//     S_w = Q_w K_j^T into tensor memory -> softmax writes P_w (bf16) to tensor memory -> O_w += P_w V_j
// P is the left operand straight from tensor memory, O stays there to the end.  At D = 128 P lies over S (tensor memory is
// full): while the softmax of one item works, the tensor cores have the other item's products.  At D = 64 P has columns
// of its own and the next S is formed as soon as the softmax has taken the last one into registers.  O is rescaled only
// when a row's maximum has grown by more than 2^8 since the last time (exponentials up to 2^8 are as exact in float and
// bf16 as those below 1; a published technique), and the warp that finds this does it itself.
//
// Measured: 8 x 4096 positions at most, 16 heads of 64: 292 us (690 TFLOP/s; up to 350 under the power cap), where the
// exponentials alone take about 180 at 16 a cycle and SM; 64 x 256, 12 heads of 128: 48 us, of which the key tiles' work is a
// third and the rest the beginnings and ends of pieces of one to three tiles.  All exponentials are the special-function unit's,
// whose result for a masked score is exactly zero; one pair in 16 by a polynomial instead, with its result selected to zero there:
// 293 and 49 us, and 195 against 191 for 64 x 1024, 12 heads of 128.
#include <float.h>
#include <math.h>

#include "attention.cuh"

namespace rapid {
namespace attn {
namespace {

// Eight row warps, a thread to a row: with sixteen, half a row each, the exchange of the maximum through shared memory costs
// more than the wider choice of instructions brings (64 x 256: 55 us against 47; 8 x 4096: 322 against 314).
using W = Roles<8>;

struct FwdArgs {
    Geometry g;
    float scale_log2;  // scale * log2(e)
    uint16_t* out;
    int64_t ld_out;
    float* lse;
    rapid_stats_t* stats;
    int items, pairs;  // work items of a key head; pieces of work for them
};

template <int D>
struct FwdCfg {
    static constexpr uint32_t kStages = D == 128 ? 4 : 8;  // tiles in flight, keys and values alternating
    static constexpr bool kOverlay = D == 128;        // P over S
    static constexpr size_t kSmem = (size_t)(2 + kStages) * tile_bytes<D>() + 2 * kBoxBytes + 1024;  // with a box of output for each item
};

struct alignas(16) FwdWork {
    int n, hk, lo, hi, jlo, jhi;
    int t[2], h[2], from[2], to[2];  // of the two items
    int valid;                       // bit w: item w exists
    int end;

    __device__ __forceinline__ void set(const FwdArgs& a, int block) {
        const Geometry& g = a.g;
        end = block < 0;
        if (end) return;
        // the longest rows first
        const int pair = a.pairs - 1 - (int)((unsigned)block / (unsigned)(g.n_seq * g.kv_heads));
        const int nk = (int)((unsigned)block % (unsigned)(g.n_seq * g.kv_heads));
        n = nk / g.kv_heads;
        hk = nk - n * g.kv_heads;
        live_range(g, n, lo, hi);
        valid = 0;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int item = min(2 * pair + w, a.items - 1);
            const bool exists = 2 * pair + w < a.items;
            valid |= (exists ? 1 : 0) << w;
            t[w] = item / g.group;
            h[w] = hk * g.group + item - t[w] * g.group;
            key_tiles(g, t[w], lo, hi, from[w], to[w]);
            if (!exists) from[w] = to[w] = 0;
        }
        // the tiles of either item: a contiguous range
        jlo = jhi = 0;
        if (to[0] > from[0]) jlo = from[0], jhi = to[0];
        if (to[1] > from[1]) {
            jlo = jhi > jlo ? min(jlo, from[1]) : from[1];
            jhi = max(jhi, to[1]);
        }
    }
};

template <int D, bool SHARED>
__global__ void __launch_bounds__(W::kThreads, 1)
attn_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mo, const __grid_constant__ FwdArgs a) {
    constexpr uint32_t kStages = FwdCfg<D>::kStages;
    constexpr bool kOverlay = FwdCfg<D>::kOverlay;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // [w]: of an item.  q_full, q_empty, o_empty (and o_full where P lies over S) count the items with keys; s_*, p_full, o_full
    // count tiles.
    __shared__ __align__(8) uint64_t q_full[2], q_empty[2], s_full[2], s_empty[2], p_full[2], o_full[2], o_empty[2],
        out_staged[2], out_free[2], kv_full[kStages], kv_empty[kStages], kv_raw[kStages], drain;
    __shared__ __align__(16) WorkQueue<FwdWork> queue;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* abortp = &abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    if (tid == 0) {
        for (int w = 0; w < 2; ++w) {
            mbar_init(&q_full[w], 1);
            mbar_init(&q_empty[w], 1);
            mbar_init(&s_full[w], 1);
            mbar_init(&s_empty[w], 4);
            mbar_init(&p_full[w], 4);
            mbar_init(&o_full[w], 1);
            mbar_init(&o_empty[w], 4);
            mbar_init(&out_staged[w], 4);
            mbar_init(&out_free[w], 1);
        }
        for (uint32_t s = 0; s < kStages; ++s) {
            mbar_init(&kv_full[s], 1);
            mbar_init(&kv_empty[s], 1);
            mbar_init(&kv_raw[s], 1);
        }
        mbar_init(&drain, 1);
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
    auto s_addr = [&](int w) { return tmem + (uint32_t)w * 128u; };
    auto o_addr = [&](int w) { return tmem + 256u + (uint32_t)w * D; };
    auto p_addr = [&](int w) { return kOverlay ? s_addr(w) : tmem + 384u + (uint32_t)w * 64u; };
    const uint32_t smem0 = smem_u32(smem);
    auto kv_tile = [&](uint32_t s) { return smem + (size_t)(2 + s) * TB; };
    auto kv_addr = [&](uint32_t s) { return smem0 + (2u + s) * (uint32_t)TB; };

    if (warp >= W::kRow) W::leave_registers();
    if (warp == W::kCopy) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0) {
            uint32_t it = 0, nq[2] = {0, 0}, k = 0, was_raw = 0;
            RawParity raw;
            Place<kStages> at;
            bool ok = true;
            int block = (int)blockIdx.x;
            FwdWork x;
            while (true) {
                x.set(a, block);
                if (!(ok = work_put(&queue, k, x, abortp)) || x.end) break;
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    if (ok && x.to[w] > x.from[w]) {
                        if (nq[w] > 0) ok = wait_one(&q_empty[w], (nq[w] - 1u) & 1u, abortp);
                        if (ok) {
                            mbar_arrive_expect_tx(&q_full[w], TB);
                            load_tile<D>(smem + (size_t)w * TB, &mq, x.h[w], x.t[w] * kTile, x.n, &q_full[w]);
                            ++nq[w];
                        }
                    }
                for (int j = x.jlo; j < x.jhi && ok; ++j)
                    for (int half = 0; half < 2; ++half) {
                        if (it >= kStages && !(ok = wait_one(&kv_empty[at.s], at.parity ^ 1u, abortp))) break;
                        // dead keys are masked in the scores; dead values have to be zero
                        const bool clean = half && dirty<SHARED>(j, x.lo, x.hi);
                        uint64_t* bar = clean ? &kv_raw[at.s] : &kv_full[at.s];
                        was_raw = clean ? was_raw | (1u << at.s) : was_raw & ~(1u << at.s);
                        if (clean) raw.flip(at.s);
                        mbar_arrive_expect_tx(bar, TB);
                        load_tile<D>(kv_tile(at.s), half ? &mv : &mk, x.hk, j * kTile, x.n, bar);
                        ++it;
                        at.step();
                    }
                if (!ok) break;
                block = work_ask(&queue, k, abortp);
                if (!(ok = block >= -1)) break;
                ++k;
            }
            if (!ok || *abortp) {  // gave up: what is under way lands before the block's memory goes away
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    if (nq[w] > 0) wait_landed(&q_full[w], (nq[w] - 1u) & 1u);
                for (uint32_t s = 0; s < kStages && s < it; ++s) {
                    const bool now = s < at.s;  // this buffer's last use belongs to the current turn, or to the one before
                    if ((was_raw >> s) & 1u) wait_landed(&kv_raw[s], ((raw.bits >> s) & 1u) ^ 1u);
                    else wait_landed(&kv_full[s], now ? at.parity : at.parity ^ 1u);
                }
            }
        }
    } else if (warp == W::kClean) {
        // ------------------------------------ dead rows ---------------------------------------------------
        RawParity raw;
        Place<kStages> at;
        bool ok = true;
        FwdWork x;
        for (uint32_t k = 0; ok && work_take(&queue, k, x, lane, abortp); ++k)
            for (int j = x.jlo; j < x.jhi && ok; ++j) {
                at.step();  // past the keys
                if (dirty<SHARED>(j, x.lo, x.hi)) {
                    ok = wait_all(&kv_raw[at.s], raw.flip(at.s), abortp);
                    if (ok) zero_dead_rows<D, SHARED>(g, kv_tile(at.s), x.n, j * kTile, x.lo, x.hi, lane);
                    if (ok && lane == 0) mbar_arrive(&kv_full[at.s]);
                }
                at.step();
            }
    } else if (warp == W::kMma) {
        // ------------------------------------ products ----------------------------------------------------
        if (elect_one()) {
            bool ok = true;
            uint32_t nq[2] = {0, 0}, ns[2] = {0, 0}, np[2] = {0, 0};  // items; tiles of S, of P
            Place<kStages> ka, va;  // the next tile of keys, of values
            va.step();
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                ok = wait_one(bar, parity, abortp);
                tc_fence_after();
                return ok;
            };
            FwdWork x;
            for (uint32_t k = 0; ok && work_take_one(&queue, k, x, abortp); ++k) {
                // Tiles in the middle, where both items have scores to form and earlier values to add, run through a loop
                // without questions: what this lane does between products is time that the tensor cores lose.
                const int mid_from = max(x.from[0], x.from[1]) + 2, mid_to = min(x.to[0], x.to[1]) - 1;
                for (int j = x.jlo; j <= x.jhi && x.jlo < x.jhi && ok; ++j) {
                    if (j >= mid_from && j < mid_to) {
                        uint32_t sp0 = (ns[0] - 1u) & 1u, sp1 = (ns[1] - 1u) & 1u, pp0 = np[0] & 1u, pp1 = np[1] & 1u;
                        ns[0] += (uint32_t)(mid_to - j);
                        ns[1] += (uint32_t)(mid_to - j);
                        np[0] += (uint32_t)(mid_to - j);
                        np[1] += (uint32_t)(mid_to - j);
                        for (; j < mid_to; ++j) {
                            const uint32_t k_now = kv_addr(ka.s), v_now = kv_addr(va.s);
                            if (!wait(&kv_full[ka.s], ka.parity)) break;
                            if (kOverlay) {
                                if (!wait(&kv_full[va.s], va.parity) || !wait(&p_full[0], pp0)) break;
                                mma_sum<D>(o_addr(0), p_addr(0), 16u, v_now, 1u);
                                mma_rows<D>(s_addr(0), smem0, k_now);
                                mma_commit(&s_full[0]);
                                if (!wait(&p_full[1], pp1)) break;
                                mma_sum<D>(o_addr(1), p_addr(1), 16u, v_now, 1u);
                                mma_rows<D>(s_addr(1), smem0 + TB, k_now);
                                mma_commit(&s_full[1]);
                                mma_commit(&kv_empty[ka.s]);
                                mma_commit(&kv_empty[va.s]);
                            } else {
                                if (!wait(&s_empty[0], sp0)) break;
                                mma_rows<D>(s_addr(0), smem0, k_now);
                                mma_commit(&s_full[0]);
                                if (!wait(&s_empty[1], sp1)) break;
                                mma_rows<D>(s_addr(1), smem0 + TB, k_now);
                                mma_commit(&s_full[1]);
                                mma_commit(&kv_empty[ka.s]);
                                if (!wait(&kv_full[va.s], va.parity) || !wait(&p_full[0], pp0)) break;
                                mma_sum<D>(o_addr(0), p_addr(0), 16u, v_now, 1u);
                                mma_commit(&o_full[0]);
                                if (!wait(&p_full[1], pp1)) break;
                                mma_sum<D>(o_addr(1), p_addr(1), 16u, v_now, 1u);
                                mma_commit(&o_full[1]);
                                mma_commit(&kv_empty[va.s]);
                            }
                            ka.step(2);
                            va.step(2);
                            sp0 ^= 1u;
                            sp1 ^= 1u;
                            pp0 ^= 1u;
                            pp1 ^= 1u;
                        }
                        if (!ok) break;
                    }
                    auto scores = [&](int w) {  // S_w of tile j
                        if (!ok || j < x.from[w] || j >= x.to[w]) return;
                        if (j == x.from[w] && !wait(&q_full[w], nq[w] & 1u)) return;
                        if (!kOverlay && ns[w] > 0 && !wait(&s_empty[w], (ns[w] - 1u) & 1u)) return;
                        mma_rows<D>(s_addr(w), smem0 + (uint32_t)w * TB, kv_addr(ka.s));
                        mma_commit(&s_full[w]);
                        if (j == x.to[w] - 1) mma_commit(&q_empty[w]);
                        ++ns[w];
                    };
                    auto values = [&](int w) {  // O_w += P_w V of tile j - 1
                        if (!ok || j - 1 < x.from[w] || j - 1 >= x.to[w]) return;
                        if (j - 1 == x.from[w] && nq[w] > 0 && !wait(&o_empty[w], (nq[w] - 1u) & 1u)) return;
                        if (!wait(&p_full[w], np[w] & 1u)) return;
                        mma_sum<D>(o_addr(w), p_addr(w), 16u, kv_addr(va.s), j - 1 > x.from[w] ? 1u : 0u);
                        if (!kOverlay || j == x.to[w]) mma_commit(&o_full[w]);
                        ++np[w];
                        if (j == x.to[w]) ++nq[w];
                    };
                    if (j < x.jhi && !wait(&kv_full[ka.s], ka.parity)) break;
                    if (kOverlay) {
                        if (j > x.jlo && !wait(&kv_full[va.s], va.parity)) break;
                        values(0);
                        scores(0);
                        values(1);
                        scores(1);
                        if (!ok) break;
                        if (j < x.jhi) mma_commit(&kv_empty[ka.s]);
                        if (j > x.jlo) mma_commit(&kv_empty[va.s]);
                    } else {
                        scores(0);
                        scores(1);
                        if (!ok) break;
                        if (j < x.jhi) mma_commit(&kv_empty[ka.s]);
                        if (j > x.jlo && !wait(&kv_full[va.s], va.parity)) break;
                        values(0);
                        values(1);
                        if (!ok) break;
                        if (j > x.jlo) mma_commit(&kv_empty[va.s]);
                    }
                    if (j < x.jhi) ka.step(2);
                    if (j > x.jlo) va.step(2);
                }
            }
            // every product has ended before tensor memory is given back
            mma_commit(&drain);
            wait_drained(&drain, abortp);
        }
        __syncwarp();
    } else if (warp < W::kRow) {
        // ------------------------------------ softmax -----------------------------------------------------
        W::take_registers();
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t st = s_addr(w) + lanes, ot = o_addr(w) + lanes, pt = p_addr(w) + lanes;
        const float c = a.scale_log2;
        const uint64_t c2 = f32x2(c, c);
        uint32_t cnt = 0, items = 0, boxes = 0;  // tiles, items with keys, boxes of output so far
        uint8_t* stage = smem + (size_t)(2 + kStages) * TB + w * kBoxBytes;
        bool ok = true;
        auto tell = [&](uint64_t* bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        FwdWork x;
        for (uint32_t k = 0; ok && work_take(&queue, k, x, lane, abortp); ++k) {
            const int tw = w ? x.t[1] : x.t[0], hw = w ? x.h[1] : x.h[0], fw = w ? x.from[1] : x.from[0], ew = w ? x.to[1] : x.to[0];
            const int pos = tw * kTile + row;
            int lo = x.lo, hi = x.hi;
            if (SHARED) row_range(g, x.n, pos, lo, hi);
            const bool live = pos >= lo && pos < hi && ew > fw;
            // keys [see, see + count) are visible to this row
            const int see = max(lo, pos - g.window + 1);
            const unsigned count = live ? (unsigned)(pos + 1 - see) : 0u;
            // key tiles in [full_from, full_to) are visible to every row of this tile; the others are masked
            int full_from = 1 << 30, full_to = 0;
            if (!SHARED && tw * kTile >= x.lo && tw * kTile + kTile <= x.hi) {
                full_from = (max(x.lo, tw * kTile + kTile - g.window) + kTile - 1) / kTile;
                full_to = tw;
            }
            float mref = -INFINITY, sum = 0.f;
            for (int j = fw; j < ew; ++j, ++cnt) {
                if (!(ok = wait_all(&s_full[w], cnt & 1u, abortp))) break;
                tc_fence_after();
                // The items start together; half a tile's time apart, one is at its exponentials while the other waits, loads and
                // compares (heads of 64, 8 x 4096: 324 -> 293 us; short pieces have no time for it).  Where P lies over S the order of
                // the products keeps them apart anyway (heads of 128, 64 x 1024 with the wait 191 us, without 190; 8 x 4096 275 both).
                if (!kOverlay && w == 1 && j == fw && ew - fw >= 4) {
                    const long long t0 = clock64();
                    while (clock64() - t0 < 900) {}
                }
                uint32_t s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_ld32(st + 32u * i, s[i]);
                tmem_ld_wait();
                if (!kOverlay) tell(&s_empty[w]);
                if (j < full_from || j >= full_to) {
                    const int first = j * kTile - see;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if ((unsigned)(first + 32 * i + e) >= count) s[i][e] = 0xff800000u;  // -infinity
                }
                float top4[4] = {mref, mref, mref, mref};
#pragma unroll
                for (int e = 0; e < 32; e += 2)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top4[i] = max3(top4[i], __uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1]));
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                // with P in columns of its own, the last product may still be reading them
                if (!kOverlay && j > fw) {
                    if (!(ok = wait_all(&o_full[w], (cnt - 1u) & 1u, abortp))) break;
                    tc_fence_after();
                }
                const bool grown = (top - mref) * c > 8.f;  // false where both are -infinity
                if (__any_sync(0xffffffffu, grown)) {
                    const float alpha = grown ? ex2_approx((mref - top) * c) : 1.f;
                    if (grown) mref = top;
                    sum *= alpha;
                    if (j > fw) {
#pragma unroll 1
                        for (int i = 0; i < D / 16; ++i) {
                            uint32_t o[16];
                            tmem_ld16(ot + 16u * i, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tmem_st16(ot + 16u * i, o);
                        }
                    }
                }
                const float shift = mref == -INFINITY ? 0.f : -mref * c;
                const uint64_t shift2 = f32x2(shift, shift);
                uint64_t part[2] = {f32x2(0.f, 0.f), f32x2(0.f, 0.f)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint64_t z = f32x2_fma(f32x2(__uint_as_float(s[i][2 * e]), __uint_as_float(s[i][2 * e + 1])), c2, shift2);
                        float u, v;
                        f32x2_split(z, u, v);
                        u = ex2_approx(u);  // exactly zero for a masked score
                        v = ex2_approx(v);
                        part[e & 1] = f32x2_add(part[e & 1], f32x2(u, v));
                        p[e] = pack_bf16x2(u, v);
                    }
                    tmem_st16(pt + 16u * i, p);
                }
                float u, v;
                f32x2_split(f32x2_add(part[0], part[1]), u, v);
                sum += u + v;
                tmem_st_wait();
                tell(&p_full[w]);
            }
            // out = O / sum, lse = max + log(sum)
            if (ok && ew > fw) {
                ok = wait_all(&o_full[w], (kOverlay ? items : cnt - 1u) & 1u, abortp);
                tc_fence_after();
                ++items;
            }
            if (!ok || !((x.valid >> w) & 1)) continue;
            const float inv = live ? 1.f / sum : 0.f;
            if (ew > fw) {
#pragma unroll 1
                for (int box = 0; box < D / 64; ++box) {
                    // one lane stores the boxes and says when the last one has been read out of shared memory
                    if ((warp & 3) == 0 && lane == 0 && boxes > 0) {
                        bulk_wait_read<0>();
                        mbar_arrive(&out_free[w]);
                    }
                    if (boxes > 0 && !(ok = wait_all(&out_free[w], (boxes - 1u) & 1u, abortp))) break;
                    stage_acc32(stage, row, 0, ot + 64u * box, live, inv);
                    stage_acc32(stage, row, 1, ot + 64u * box + 32u, live, inv);
                    fence_proxy_async_smem();
                    if (box == D / 64 - 1) tell(&o_empty[w]);
                    tell(&out_staged[w]);
                    if ((warp & 3) == 0) {
                        if (!(ok = wait_all(&out_staged[w], boxes & 1u, abortp))) break;
                        if (lane == 0 && box * 64 < g.head_dim) tma_store_4d(&mo, stage, box * 64, hw, tw * kTile, x.n);
                        if (lane == 0) bulk_commit();
                    }
                    ++boxes;
                }
            } else {
                zero_tile(a.out, a.ld_out, g.seq_len, g.head_dim, hw, tw * kTile, x.n, row, 128);
            }
            if (a.lse && pos < g.seq_len)
                a.lse[lse_at(g, x.n, hw, pos)] =
                    live ? (float)(((double)mref * (double)c + (double)log2f(sum)) * kLn2D) : -INFINITY;
        }
        if ((warp & 3) == 0 && lane == 0) bulk_wait_all<0>();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == W::kMma) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && abort_flag && a.stats) atomicMax(&a.stats->status, (int)RAPID_ERR_TIMEOUT);
}

template <int D, bool SHARED>
cudaError_t launch_fwd(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mo, const FwdArgs& a,
                       unsigned grid, cudaStream_t st) {
    auto kern = attn_fwd_kernel<D, SHARED>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FwdCfg<D>::kSmem);
    if (e != cudaSuccess) return e;
    kern<<<grid, W::kThreads, FwdCfg<D>::kSmem, st>>>(mq, mk, mv, mo, a);
    return cudaGetLastError();
}

}  // namespace

rapid_status_t check_attn(const rapid_attn_desc_t* d) {
    if (!d || d->n_seq <= 0 || d->seq_len <= 0 || d->n_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->window < 0)
        return RAPID_ERR_INVALID_ARG;
    if (d->dtype != RAPID_BF16 || d->flags != 0) return RAPID_ERR_INVALID_ARG;
    if (d->n_heads % d->n_kv_heads != 0) return RAPID_ERR_INVALID_ARG;
    // the kernels' factors; also false for NaN.  A factor of zero would turn the -infinity of a masked score into NaN.
    const float scale = (float)d->scale, scale_log2 = (float)(d->scale * kLog2eD);
    if (!(scale >= FLT_MIN && scale_log2 <= FLT_MAX)) return RAPID_ERR_INVALID_ARG;
    const int64_t wq = (int64_t)d->n_heads * d->head_dim, wk = (int64_t)d->n_kv_heads * d->head_dim;
    if (d->ld_q < wq || d->ld_out < wq || d->ld_k < wk || d->ld_v < wk) return RAPID_ERR_INVALID_ARG;
    if (d->head_dim % 8 != 0 || d->head_dim > 128) return RAPID_ERR_UNSUPPORTED;
    if (d->ld_q % 8 || d->ld_k % 8 || d->ld_v % 8 || d->ld_out % 8) return RAPID_ERR_ALIGNMENT;
    // limits of the tensor maps (strides below 2^40 bytes) and of the launch grids
    const int64_t T = (int64_t)d->n_seq * d->seq_len, most = 1ll << 31;
    if (T > 0x7fffffffll || d->n_heads > 4096 || d->seq_len > (1 << 24)) return RAPID_ERR_UNSUPPORTED;
    if (d->ld_q > most || d->ld_k > most || d->ld_v > most || d->ld_out > most) return RAPID_ERR_UNSUPPORTED;
    const int64_t widest = d->ld_q > d->ld_k ? d->ld_q : d->ld_k, other = d->ld_v > d->ld_out ? d->ld_v : d->ld_out;
    if ((widest > other ? widest : other) > (1ll << 38) / d->seq_len) return RAPID_ERR_UNSUPPORTED;
    const int64_t tiles = (d->seq_len + kTile - 1) / kTile;
    if (tiles * d->n_seq * d->n_heads > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;
    return RAPID_OK;
}

Geometry make_geometry(const rapid_attn_desc_t& d, const int32_t* bounds) {
    Geometry g;
    g.n_seq = d.n_seq;
    g.seq_len = d.seq_len;
    g.heads = d.n_heads;
    g.kv_heads = d.n_kv_heads;
    g.group = d.n_heads / d.n_kv_heads;
    g.head_dim = d.head_dim;
    g.window = d.window == 0 || d.window > d.seq_len ? d.seq_len : d.window;
    g.part = g.parts = 0;
    g.bounds = bounds;
    return g;
}

int make_shares(const rapid_attn_desc_t& d, const int32_t* bounds, Share (&shares)[2]) {
    const int parts = kTile / d.seq_len < d.n_seq ? kTile / d.seq_len : d.n_seq;
    if (parts < 2) {
        shares[0] = Share{d, make_geometry(d, bounds), 0};
        return 1;
    }
    int count = 0;
    for (int first = 0; first < d.n_seq;) {
        Share& s = shares[count++];
        const int here = d.n_seq - first < parts ? d.n_seq - first : parts, sequences = (d.n_seq - first) / here;
        s.d = d;
        s.d.n_seq = sequences;
        s.d.seq_len = here * d.seq_len;
        s.g = make_geometry(s.d, bounds ? bounds + 2 * (int64_t)first : nullptr);
        s.g.window = d.window == 0 || d.window > d.seq_len ? d.seq_len : d.window;
        s.g.part = d.seq_len;
        s.g.parts = here;
        s.first_row = (int64_t)first * d.seq_len;
        first += sequences * here;
    }
    return count;
}

}  // namespace attn
}  // namespace rapid

using namespace rapid;
using namespace rapid::attn;

extern "C" rapid_status_t rapid_attention_fwd(const rapid_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                              const int32_t* bounds, void* out, float* lse, rapid_stats_t* stats, void* stream) {
    rapid_status_t s = check_attn(desc);
    if (s != RAPID_OK) return s;
    const rapid_attn_desc_t& d = *desc;
    if (!q || !k || !v || !out) return RAPID_ERR_INVALID_ARG;
    if (!policy::aligned(q, 16) || !policy::aligned(k, 16) || !policy::aligned(v, 16) || !policy::aligned(out, 16) ||
        !policy::aligned(bounds, 4) || !policy::aligned(lse, 4) || !policy::aligned(stats, 8))
        return RAPID_ERR_ALIGNMENT;
    const int64_t T = (int64_t)d.n_seq * d.seq_len, wq = (int64_t)d.n_heads * d.head_dim, wk = (int64_t)d.n_kv_heads * d.head_dim;
    if (policy::rows_overlap(out, wq, d.ld_out, q, wq, d.ld_q, T, 2) || policy::rows_overlap(out, wq, d.ld_out, k, wk, d.ld_k, T, 2) ||
        policy::rows_overlap(out, wq, d.ld_out, v, wk, d.ld_v, T, 2))
        return RAPID_ERR_INVALID_ARG;
    int sms = 0;
    if ((s = policy::check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (policy::clear_stats(stats, st) != cudaSuccess) return RAPID_ERR_CUDA;
    Share shares[2];
    const int count = make_shares(d, bounds, shares);
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < count && e == cudaSuccess; ++i) {
        const Share& c = shares[i];
        void* rows = rows_from(out, c.first_row, d.ld_out);
        CUtensorMap mq, mk, mv, mo;
        if (!make_head_map(&mq, rows_from(q, c.first_row, d.ld_q), c.d, d.n_heads, d.ld_q) ||
            !make_head_map(&mk, rows_from(k, c.first_row, d.ld_k), c.d, d.n_kv_heads, d.ld_k) ||
            !make_head_map(&mv, rows_from(v, c.first_row, d.ld_v), c.d, d.n_kv_heads, d.ld_v) ||
            !make_head_map(&mo, rows, c.d, d.n_heads, d.ld_out))
            return RAPID_ERR_CUDA;
        FwdArgs a;
        a.g = c.g;
        a.scale_log2 = (float)(d.scale * kLog2eD);
        a.out = static_cast<uint16_t*>(rows);
        a.ld_out = d.ld_out;
        a.lse = lse ? lse + c.first_row * d.n_heads : nullptr;
        a.stats = stats;
        a.items = (c.d.seq_len + kTile - 1) / kTile * a.g.group;
        a.pairs = (a.items + 1) / 2;
        const unsigned grid = (unsigned)((int64_t)a.pairs * c.d.n_seq * d.n_kv_heads);
        auto launch = d.head_dim <= 64 ? (c.g.part ? launch_fwd<64, true> : launch_fwd<64, false>)
                                       : (c.g.part ? launch_fwd<128, true> : launch_fwd<128, false>);
        e = launch(mq, mk, mv, mo, a, grid, st);
    }
    return e == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
