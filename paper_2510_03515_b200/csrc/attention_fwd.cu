// Causal attention, forward (tcgen05).
//
// A block takes two work items of one key head: an item is (query tile of 128 positions, query head of the group), items
// are numbered tile by tile, so the two usually share the tile and always the keys.  Warps 0-3 and 4-7 each run the
// softmax of one item, a thread to a row, so row maximum and sum need no exchange; warp 8 issues the copies, warp 9 the
// products:
//     S_w = Q_w K_j^T into tensor memory -> softmax reads it, writes P_w (bf16) over it -> O_w += P_w V_j
// P is the left operand straight from tensor memory, O stays there to the end.  While the softmax of one item works, the
// tensor cores have the other item's products, so neither waits long.  O is rescaled only when a row's maximum has grown
// by more than 2^8 since the last time (exponentials up to 2^8 are as exact in float and bf16 as those below 1), and the
// warp that finds this does it itself: the barrier that says "S of this tile is there" also says that every earlier
// product has ended.
#include <math.h>

#include "attention.cuh"

namespace rapid {
namespace attn {
namespace {

constexpr int kThreads = 320;

struct FwdArgs {
    Geometry g;
    float scale_log2;  // scale * log2(e)
    float* lse;
    rapid_stats_t* stats;
    int items, pairs;  // work items of a key head; blocks for them
};

template <int D>
struct FwdCfg {
    static constexpr int kStages = D == 128 ? 4 : 8;  // tiles of keys and values in flight
    static constexpr size_t kSmem = (size_t)(2 + kStages) * tile_bytes<D>() + 1024;
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attn_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mo, FwdArgs a) {
    constexpr int kStages = FwdCfg<D>::kStages;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t q_full[2], s_full[2], p_full[2], o_full[2], kv_full[kStages], kv_empty[kStages], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* abortp = &abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    // the longest rows first
    const int pair = a.pairs - 1 - (int)(blockIdx.x / (unsigned)(g.n_seq * g.kv_heads));
    const int nk = (int)(blockIdx.x % (unsigned)(g.n_seq * g.kv_heads));
    const int n = nk / g.kv_heads, hk = nk - n * g.kv_heads;
    int lo, hi;
    live_range(g, n, lo, hi);
    int t[2], h[2], from[2], to[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int item = min(2 * pair + w, a.items - 1);
        t[w] = item / g.group;
        h[w] = hk * g.group + item - t[w] * g.group;
        key_tiles(g, t[w], lo, hi, from[w], to[w]);
        if (2 * pair + w >= a.items) from[w] = to[w] = 0;
    }
    // tiles of either item, a contiguous range
    int jlo = 0, jhi = 0;
    if (to[0] > from[0]) jlo = from[0], jhi = to[0];
    if (to[1] > from[1]) {
        jlo = jhi > jlo ? min(jlo, from[1]) : from[1];
        jhi = max(jhi, to[1]);
    }

    if (tid == 0) {
        for (int w = 0; w < 2; ++w) {
            mbar_init(&q_full[w], 1);
            mbar_init(&s_full[w], 1);
            mbar_init(&p_full[w], 4);
            mbar_init(&o_full[w], 1);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&kv_full[s], 1);
            mbar_init(&kv_empty[s], 1);
        }
        mbar_init(&drain, 1);
        abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == 9) {
        tmem_alloc(&tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    auto s_addr = [&](int w) { return tmem + (uint32_t)w * 128u; };
    auto o_addr = [&](int w) { return tmem + 256u + (uint32_t)w * D; };
    auto kv_tile = [&](uint32_t it) { return smem + (size_t)(2 + it % kStages) * TB; };

    if (warp == 8) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0) {
#pragma unroll
            for (int w = 0; w < 2; ++w)
                if (to[w] > from[w]) {
                    mbar_arrive_expect_tx(&q_full[w], TB);
                    load_tile<D>(smem + (size_t)w * TB, &mq, h[w], t[w] * kTile, n, &q_full[w]);
                }
            uint32_t it = 0;
            bool ok = true;
            for (int j = jlo; j < jhi && ok; ++j)
                for (int half = 0; half < 2; ++half, ++it) {
                    const int s = it % kStages;
                    const uint32_t use = it / kStages;
                    if (use > 0 && !mbar_wait_bounded(&kv_empty[s], (use & 1u) ^ 1u, abortp)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(&kv_full[s], TB);
                    load_tile<D>(kv_tile(it), half ? &mv : &mk, hk, j * kTile, n, &kv_full[s]);
                }
            if (!ok || *abortp) {  // gave up: let the copies land before the block's memory goes away
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    if (to[w] > from[w]) {
                        const unsigned long long t0 = global_timer_ns();
                        while (!mbar_try_wait(&q_full[w], 0))
                            if (global_timer_ns() - t0 > kWaitLimitNs) break;
                    }
                for (uint32_t i = it > (uint32_t)kStages ? it - kStages : 0u; i < it; ++i) {
                    const unsigned long long t0 = global_timer_ns();
                    while (!mbar_try_wait(&kv_full[i % kStages], (i / kStages) & 1u))
                        if (global_timer_ns() - t0 > kWaitLimitNs) break;
                }
            }
        }
    } else if (warp == 9) {
        // ------------------------------------ products ----------------------------------------------------
        // All lanes walk the loop (they clear dead rows together); lane 0 issues.
        bool ok = true;
        uint32_t done[2] = {0, 0};  // tiles of P consumed
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abortp));
            return ok;
        };
        for (int j = jlo; j <= jhi && jlo < jhi && ok; ++j) {
            const uint32_t itk = 2u * (uint32_t)(j - jlo), itv = itk - 1u;  // ring numbers of K_j and V_{j-1}
            if (j < jhi && !wait(&kv_full[itk % kStages], (itk / kStages) & 1u)) break;
            if (j > jlo) {
                if (!wait(&kv_full[itv % kStages], (itv / kStages) & 1u)) break;
                zero_rows_outside<D>(kv_tile(itv), (j - 1) * kTile, lo, hi, lane);
            }
            tc_fence_after();
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (j - 1 >= from[w] && j - 1 < to[w]) {
                    if (!wait(&p_full[w], done[w] & 1u)) break;
                    tc_fence_after();
                    if (lane == 0) {
                        const uint32_t v = smem_u32(kv_tile(itv));
#pragma unroll
                        for (int ks = 0; ks < kTile / 16; ++ks)
                            mma_f16_ts(o_addr(w), s_addr(w) + 8u * ks, desc_mn(v, ks), instr_desc(D, true), (done[w] | ks) ? 1u : 0u);
                        mma_commit(&o_full[w]);
                    }
                    ++done[w];
                }
                if (j >= from[w] && j < to[w]) {
                    if (j == from[w] && !wait(&q_full[w], 0)) break;
                    tc_fence_after();
                    if (lane == 0) {
                        mma_ss<D>(s_addr(w), smem_u32(smem + (size_t)w * TB), smem_u32(kv_tile(itk)));
                        mma_commit(&s_full[w]);
                    }
                }
            }
            if (!ok) break;
            if (lane == 0) {
                if (j < jhi) mma_commit(&kv_empty[itk % kStages]);
                if (j > jlo) mma_commit(&kv_empty[itv % kStages]);
            }
        }
        if (lane == 0) {  // every product has ended before tensor memory is given back
            mma_commit(&drain);
            const unsigned long long t0 = global_timer_ns();
            while (!mbar_try_wait(&drain, 0))
                if (global_timer_ns() - t0 > kWaitLimitNs) {
                    *abortp = 1;
                    break;
                }
        }
    } else {
        // ------------------------------------ softmax -----------------------------------------------------
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const int tw = w ? t[1] : t[0], hw = w ? h[1] : h[0], fw = w ? from[1] : from[0], ew = w ? to[1] : to[0];
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t st = s_addr(w) + lanes, ot = o_addr(w) + lanes;
        const int pos = tw * kTile + row;
        const bool live = pos >= lo && pos < hi && ew > fw;
        // keys [see, see + count) are visible to this row
        const int see = max(lo, pos - g.window + 1);
        const unsigned count = live ? (unsigned)(pos + 1 - see) : 0u;
        // key tiles in [full_from, full_to) are visible to every row of this tile; the others are masked
        int full_from = 1 << 30, full_to = 0;
        if (tw * kTile >= lo && tw * kTile + kTile <= hi) {
            full_from = (max(lo, tw * kTile + kTile - g.window) + kTile - 1) / kTile;
            full_to = tw;
        }
        const float c = a.scale_log2;
        float mref = -INFINITY, sum = 0.f;
        bool ok = true;
        uint32_t it = 0;
        for (int j = fw; j < ew; ++j, ++it) {
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(&s_full[w], it & 1u, abortp));
            if (!ok) break;
            tc_fence_after();
            uint32_t s[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld32(st + 32u * i, s[i]);
            tmem_ld_wait();
            if (j < full_from || j >= full_to) {
                const int first = j * kTile - see;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if ((unsigned)(first + 32 * i + k) >= count) s[i][k] = 0xff800000u;  // -infinity
            }
            float top = mref;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 32; ++k) top = fmaxf(top, __uint_as_float(s[i][k]));
            const bool grown = (top - mref) * c > 8.f;  // false where both are -infinity
            if (__any_sync(0xffffffffu, grown)) {
                const float alpha = grown ? ex2_approx((mref - top) * c) : 1.f;
                if (grown) mref = top;
                sum *= alpha;
                if (it > 0) {
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t o[32];
                        tmem_ld32(ot + 32u * i, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                        tmem_st32(ot + 32u * i, o);
                    }
                }
            }
            const float shift = mref == -INFINITY ? 0.f : -mref * c;
            const uint64_t c2 = f32x2(c, c), shift2 = f32x2(shift, shift);
            uint64_t part = f32x2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t p[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    float x, y;
                    f32x2_split(f32x2_fma(f32x2(__uint_as_float(s[i][2 * k]), __uint_as_float(s[i][2 * k + 1])), c2, shift2), x, y);
                    x = ex2_approx(x);
                    y = ex2_approx(y);
                    part = f32x2_add(part, f32x2(x, y));
                    p[k] = pack_bf16x2(x, y);
                }
                tmem_st16(st + 16u * i, p);
            }
            float x, y;
            f32x2_split(part, x, y);
            sum += x + y;
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[w]);
        }
        // out = O / sum, lse = max + log(sum).  The barrier is passed by all four warps whatever they have seen.
        if (2 * pair + w < a.items) {
            if (ew > fw && ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&o_full[w], (it - 1u) & 1u, abortp));
            tc_fence_after();
            uint8_t* stage = smem + (size_t)w * TB;  // the query tile has been read for the last time
            if (ok) {
                const float inv = live ? 1.f / sum : 0.f;
#pragma unroll 1
                for (int i = 0; i < D / 32; ++i) {
                    float f[32];
                    if (ew > fw) {
                        uint32_t o[32];
                        tmem_ld32(ot + 32u * i, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) f[k] = live ? __uint_as_float(o[k]) * inv : 0.f;
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) f[k] = 0.f;
                    }
                    stage_row32(stage, row, i, f);
                }
                if (a.lse && pos < g.seq_len)
                    a.lse[((size_t)n * g.heads + hw) * g.seq_len + pos] =
                        live ? (float)(((double)mref * (double)c + (double)log2f(sum)) * kLn2D) : -INFINITY;
                fence_proxy_async_smem();
            }
            named_barrier(1 + w, 128);
            if ((warp & 3) == 0 && lane == 0 && !*abortp) {
                store_tile<D>(&mo, stage, g.head_dim, hw, tw * kTile, n);
                bulk_commit();
                bulk_wait_all<0>();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && abort_flag && a.stats) atomicMax(&a.stats->status, (int)RAPID_ERR_TIMEOUT);
}

template <int D>
cudaError_t launch_fwd(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mo, const FwdArgs& a,
                       unsigned grid, cudaStream_t st) {
    auto kern = attn_fwd_kernel<D>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FwdCfg<D>::kSmem);
    if (e != cudaSuccess) return e;
    kern<<<grid, kThreads, FwdCfg<D>::kSmem, st>>>(mq, mk, mv, mo, a);
    return cudaGetLastError();
}

}  // namespace

rapid_status_t check_attn(const rapid_attn_desc_t* d) {
    if (!d || d->n_seq <= 0 || d->seq_len <= 0 || d->n_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->window < 0)
        return RAPID_ERR_INVALID_ARG;
    if (d->dtype != RAPID_BF16 || d->flags != 0) return RAPID_ERR_INVALID_ARG;
    if (d->n_heads % d->n_kv_heads != 0 || !(d->scale > 0.0) || !isfinite(d->scale)) return RAPID_ERR_INVALID_ARG;
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
    g.bounds = bounds;
    return g;
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
    if (!policy::aligned(q, 16) || !policy::aligned(k, 16) || !policy::aligned(v, 16) || !policy::aligned(out, 16))
        return RAPID_ERR_ALIGNMENT;
    const int64_t T = (int64_t)d.n_seq * d.seq_len, wq = (int64_t)d.n_heads * d.head_dim, wk = (int64_t)d.n_kv_heads * d.head_dim;
    if (policy::rows_overlap(out, wq, d.ld_out, q, wq, d.ld_q, T, 2) || policy::rows_overlap(out, wq, d.ld_out, k, wk, d.ld_k, T, 2) ||
        policy::rows_overlap(out, wq, d.ld_out, v, wk, d.ld_v, T, 2))
        return RAPID_ERR_INVALID_ARG;
    int sms = 0;
    if ((s = policy::check_device(&sms)) != RAPID_OK) return s;
    CUtensorMap mq, mk, mv, mo;
    if (!make_head_map(&mq, q, d, d.n_heads, d.ld_q) || !make_head_map(&mk, k, d, d.n_kv_heads, d.ld_k) ||
        !make_head_map(&mv, v, d, d.n_kv_heads, d.ld_v) || !make_head_map(&mo, out, d, d.n_heads, d.ld_out))
        return RAPID_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (policy::clear_stats(stats, st) != cudaSuccess) return RAPID_ERR_CUDA;
    FwdArgs a;
    a.g = make_geometry(d, bounds);
    a.scale_log2 = (float)(d.scale * kLog2eD);
    a.lse = lse;
    a.stats = stats;
    a.items = (d.seq_len + kTile - 1) / kTile * a.g.group;
    a.pairs = (a.items + 1) / 2;
    const unsigned grid = (unsigned)((int64_t)a.pairs * d.n_seq * d.n_kv_heads);
    const cudaError_t e = d.head_dim <= 64 ? launch_fwd<64>(mq, mk, mv, mo, a, grid, st) : launch_fwd<128>(mq, mk, mv, mo, a, grid, st);
    return e == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
