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
// In both main kernels warps 0-7 hold 64 columns of a row each thread, warp 8 issues copies, warp 9 products.  The order of
// the products is such that the tensor cores have two products (1024 cycles at D = 128) to work on while the exponentials
// of one step are formed, and two more during its dS.
#include <math.h>

#include "attention.cuh"

namespace rapid {
namespace attn {
namespace {

constexpr int kThreads = 320;
constexpr int kVecBytes = kTile * 4;  // one float for each position of a tile

struct BwdArgs {
    Geometry g;
    float scale, scale_log2;
    int tiles;         // of a generation
    const float* shift;   // [n_seq][heads][tiles * 128]: -lse in base 2
    const float* ndelta;  // the same: -delta
    rapid_stats_t* stats;
};

// ---- row terms --------------------------------------------------------------------------------------------------

// `lanes` = 2^lanes_log2 lanes take one head of one position, 8 elements each.
__global__ void __launch_bounds__(256)
attn_row_terms_kernel(Geometry g, int tiles, int lanes_log2, const uint16_t* __restrict__ out, int64_t ld_out,
                      const uint16_t* __restrict__ dout, int64_t ld_dout, const float* __restrict__ lse, float* __restrict__ shift,
                      float* __restrict__ ndelta) {
    const int64_t padded = (int64_t)tiles * kTile;
    const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> lanes_log2;
    const int u = threadIdx.x & ((1 << lanes_log2) - 1);
    const int64_t row = unit / g.heads;  // n * padded + t
    const int h = (int)(unit - row * g.heads);
    const int n = (int)(row / padded), t = (int)(row - n * padded);
    bool live = n < g.n_seq && t < g.seq_len;
    if (live) {
        int lo, hi;
        live_range(g, n, lo, hi);
        live = t >= lo && t < hi;
    }
    float sum = 0.f;
    if (live && u * 8 < g.head_dim) {
        const int64_t r = (int64_t)n * g.seq_len + t;
        policy::Vec8<uint16_t> a, b;
        a.load(out + r * ld_out + h * g.head_dim + u * 8);
        b.load(dout + r * ld_dout + h * g.head_dim + u * 8);
        float x[8], y[8];
        a.get(x);
        b.get(y);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * y[j];
    }
    for (int o = 1; o < (1 << lanes_log2); o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (u == 0 && n < g.n_seq) {
        const int64_t at = ((int64_t)n * g.heads + h) * padded + t;
        // double: lse * log2(e) in float would shift every score of the row by its own rounding
        shift[at] = live ? (float)((double)lse[((int64_t)n * g.heads + h) * g.seq_len + t] * -kLog2eD) : -INFINITY;
        ndelta[at] = -sum;
    }
}

// ---- dK, dV -----------------------------------------------------------------------------------------------------

template <int D>
struct DkvCfg {
    static constexpr int kStages = D == 128 ? 4 : 8;  // tiles of q and dout in flight, alternating
    static constexpr size_t kSmem = (size_t)(2 + kStages) * tile_bytes<D>() + (size_t)kStages * kVecBytes + 1024;
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attn_dkv_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
                const __grid_constant__ CUtensorMap mdk, const __grid_constant__ CUtensorMap mdv, BwdArgs a) {
    constexpr int kStages = DkvCfg<D>::kStages;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t kv_full, s_full, dp_full, p_full, ds_full, all_done, full[kStages], empty[kStages];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* abortp = &abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    // the first key tiles are seen by the most queries: they go first
    const int kt = (int)(blockIdx.x / (unsigned)(g.n_seq * g.kv_heads));
    const int nk = (int)(blockIdx.x % (unsigned)(g.n_seq * g.kv_heads));
    const int n = nk / g.kv_heads, hk = nk - n * g.kv_heads;
    int lo, hi;
    live_range(g, n, lo, hi);
    const int key_last = min(kt * kTile + kTile, hi) - 1;
    int q_from = 0, q_tiles = 0;
    if (max(kt * kTile, lo) <= key_last) {
        q_from = kt;
        const int64_t last = min((int64_t)hi - 1, (int64_t)key_last + g.window - 1);
        q_tiles = (int)(last / kTile) + 1 - kt;
    }
    const int steps = q_tiles * g.group;  // step i: head hk * group + i / q_tiles, query tile q_from + i % q_tiles

    if (tid == 0) {
        mbar_init(&kv_full, 1);
        mbar_init(&s_full, 1);
        mbar_init(&dp_full, 1);
        mbar_init(&p_full, 8);
        mbar_init(&ds_full, 8);
        mbar_init(&all_done, 1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
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
    const uint32_t s_t = tmem, dp_t = tmem + 128u, dv_t = tmem + 256u, dk_t = tmem + 256u + D;
    uint8_t* k_tile = smem;
    uint8_t* v_tile = smem + TB;
    // ring number 2 i is the query tile of step i, 2 i + 1 its dout tile; both row terms come and go with the query tile,
    // which is released after the step's last reader of either (dS, then dK)
    auto tile_of = [&](uint32_t it) { return smem + (size_t)(2 + it % kStages) * TB; };
    auto vec_of = [&](uint32_t it) { return reinterpret_cast<float*>(smem + (size_t)(2 + kStages) * TB) + (it % kStages) * kTile; };

    if (warp == 8) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0 && steps > 0) {
            mbar_arrive_expect_tx(&kv_full, 2 * TB);
            load_tile<D>(k_tile, &mk, hk, kt * kTile, n, &kv_full);
            load_tile<D>(v_tile, &mv, hk, kt * kTile, n, &kv_full);
            bool ok = true;
            uint32_t it = 0;
            for (int i = 0; i < steps && ok; ++i) {
                const int h = hk * g.group + i / q_tiles, qt = q_from + i % q_tiles;
                const size_t at = (((size_t)n * g.heads + h) * a.tiles + qt) * kTile;
                for (int half = 0; half < 2; ++half, ++it) {
                    const int s = it % kStages;
                    const uint32_t use = it / kStages;
                    if (use > 0 && !mbar_wait_bounded(&empty[s], (use & 1u) ^ 1u, abortp)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(&full[s], half ? TB : TB + 2 * kVecBytes);
                    load_tile<D>(tile_of(it), half ? &mdo : &mq, h, qt * kTile, n, &full[s]);
                    if (!half) {
                        bulk_load(vec_of(it), a.shift + at, kVecBytes, &full[s]);
                        bulk_load(vec_of(it) + kTile, a.ndelta + at, kVecBytes, &full[s]);
                    }
                }
            }
            if (!ok || *abortp) {  // gave up: let the copies land before the block's memory goes away
                for (uint32_t x = it > (uint32_t)kStages ? it - kStages : 0u; x <= it; ++x) {
                    uint64_t* bar = x < it ? &full[x % kStages] : &kv_full;
                    const uint32_t parity = x < it ? (x / kStages) & 1u : 0u;
                    const unsigned long long t0 = global_timer_ns();
                    while (!mbar_try_wait(bar, parity))
                        if (global_timer_ns() - t0 > kWaitLimitNs) break;
                }
            }
        }
    } else if (warp == 9) {
        // ------------------------------------ products ----------------------------------------------------
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abortp));
            tc_fence_after();
            return ok;
        };
        // wait for a tile of the ring and clear its dead rows
        auto take = [&](uint32_t it) {
            if (!wait(&full[it % kStages], (it / kStages) & 1u)) return false;
            const int qt = q_from + (int)(it >> 1) % q_tiles;
            zero_rows_outside<D>(tile_of(it), qt * kTile, lo, hi, lane);
            return true;
        };
        // acc (+)= M (128 x 128 bf16 in tensor memory: 64 columns of a half in 32 of its own) * tile (MN-major)
        auto mma_acc = [&](uint32_t acc, uint32_t m, uint32_t tile, bool more) {
#pragma unroll
            for (int ks = 0; ks < kTile / 16; ++ks)
                mma_f16_ts(acc, m + (ks >> 2) * 64u + (ks & 3) * 8u, desc_mn(tile, ks), instr_desc(D, true), (more || ks) ? 1u : 0u);
        };
        if (steps > 0 && wait(&kv_full, 0)) {
            const uint32_t kb = smem_u32(k_tile), vb = smem_u32(v_tile);
            if (take(0) && lane == 0) {
                mma_ss<D>(s_t, kb, smem_u32(tile_of(0)));
                mma_commit(&s_full);
            }
            if (ok && take(1) && lane == 0) {
                mma_ss<D>(dp_t, vb, smem_u32(tile_of(1)));
                mma_commit(&dp_full);
            }
            for (int i = 0; i < steps && ok; ++i) {
                const uint32_t iq = 2u * i, id = iq + 1u;
                if (!wait(&p_full, i & 1)) break;
                if (lane == 0) {
                    mma_acc(dv_t, s_t, smem_u32(tile_of(id)), i > 0);
                    mma_commit(&empty[id % kStages]);
                }
                if (i + 1 < steps) {
                    if (!take(iq + 2)) break;
                    if (lane == 0) {
                        mma_ss<D>(s_t, kb, smem_u32(tile_of(iq + 2)));
                        mma_commit(&s_full);
                    }
                }
                if (!wait(&ds_full, i & 1)) break;
                if (lane == 0) {
                    mma_acc(dk_t, dp_t, smem_u32(tile_of(iq)), i > 0);
                    mma_commit(&empty[iq % kStages]);
                }
                if (i + 1 < steps) {
                    if (!take(id + 2)) break;
                    if (lane == 0) {
                        mma_ss<D>(dp_t, vb, smem_u32(tile_of(id + 2)));
                        mma_commit(&dp_full);
                    }
                }
            }
        }
        __syncwarp();
        if (lane == 0) {  // every product has ended before results are read and tensor memory is given back
            mma_commit(&all_done);
            const unsigned long long t0 = global_timer_ns();
            while (!mbar_try_wait(&all_done, 0))
                if (global_timer_ns() - t0 > kWaitLimitNs) {
                    *abortp = 1;
                    break;
                }
        }
    } else {
        // ------------------------------------ probabilities, dS -------------------------------------------
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mine = lanes + (uint32_t)half * 64u;
        const int key = kt * kTile + row;
        const float c = a.scale_log2;
        const uint64_t c2 = f32x2(c, c);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abortp));
            tc_fence_after();
            return ok;
        };
        for (int i = 0; i < steps; ++i) {
            const uint32_t iq = 2u * i;
            const int q0 = (q_from + i % q_tiles) * kTile;
            float p[64];
            if (!wait(&full[iq % kStages], (iq / kStages) & 1u) || !wait(&s_full, i & 1)) break;
            {
                uint32_t s[2][32];
                tmem_ld32(s_t + mine, s[0]);
                tmem_ld32(s_t + mine + 32u, s[1]);
                const ulonglong2* sh = reinterpret_cast<const ulonglong2*>(vec_of(iq) + half * 64);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const ulonglong2 l = sh[k];
                    const uint32_t* x = &s[k >> 3][(k & 7) * 4];
                    f32x2_split(f32x2_fma(f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), c2, l.x), p[4 * k], p[4 * k + 1]);
                    f32x2_split(f32x2_fma(f32x2(__uint_as_float(x[2]), __uint_as_float(x[3])), c2, l.y), p[4 * k + 2], p[4 * k + 3]);
                }
            }
#pragma unroll
            for (int k = 0; k < 64; ++k) p[k] = ex2_approx(p[k]);
            // the diagonal, and the far edge of a window
            if (q0 <= kt * kTile || q0 + kTile - 1 - kt * kTile >= g.window) {
                const int first = q0 + half * 64 - key;
#pragma unroll
                for (int k = 0; k < 64; ++k)
                    if ((unsigned)(first + k) >= (unsigned)g.window) p[k] = 0.f;
            }
            {
                uint32_t b[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) b[k] = pack_bf16x2(p[2 * k], p[2 * k + 1]);
                tmem_st32(s_t + mine, b);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full);

            if (!wait(&dp_full, i & 1)) break;
            {
                uint32_t s[2][32], b[32];
                tmem_ld32(dp_t + mine, s[0]);
                tmem_ld32(dp_t + mine + 32u, s[1]);
                const ulonglong2* nd = reinterpret_cast<const ulonglong2*>(vec_of(iq) + kTile + half * 64);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const ulonglong2 d = nd[k];
                    const uint32_t* x = &s[k >> 3][(k & 7) * 4];
                    float e, f;
                    f32x2_split(f32x2_mul(f32x2(p[4 * k], p[4 * k + 1]), f32x2_add(f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), d.x)), e, f);
                    b[2 * k] = pack_bf16x2(e, f);
                    f32x2_split(f32x2_mul(f32x2(p[4 * k + 2], p[4 * k + 3]), f32x2_add(f32x2(__uint_as_float(x[2]), __uint_as_float(x[3])), d.y)), e, f);
                    b[2 * k + 1] = pack_bf16x2(e, f);
                }
                tmem_st32(dp_t + mine, b);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ds_full);
        }
        // warps 0-3 write dV, warps 4-7 dK, through the tile in shared memory that is no longer needed
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&all_done, 0, abortp));
        tc_fence_after();
        const bool live = key >= lo && key < hi;
        const float factor = half ? a.scale : 1.f;
        uint8_t* stage = half ? k_tile : v_tile;
        const uint32_t acc = (half ? dk_t : dv_t) + lanes;
        if (ok) {
#pragma unroll 1
            for (int i = 0; i < D / 32; ++i) {
                float f[32];
                if (steps > 0) {
                    uint32_t o[32];
                    tmem_ld32(acc + 32u * i, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = live ? __uint_as_float(o[k]) * factor : 0.f;
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = 0.f;
                }
                stage_row32(stage, row, i, f);
            }
            fence_proxy_async_smem();
        }
        named_barrier(1 + half, 128);
        if ((warp & 3) == 0 && lane == 0 && !*abortp) {
            store_tile<D>(half ? &mdk : &mdv, stage, g.head_dim, hk, kt * kTile, n);
            bulk_commit();
            bulk_wait_all<0>();
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

// ---- dQ ---------------------------------------------------------------------------------------------------------

template <int D>
struct DqCfg {
    static constexpr int kKeys = 3, kVals = 2;  // tiles of keys (needed for two steps) and of values in flight
    static constexpr size_t kSmem = (size_t)(2 + kKeys + kVals) * tile_bytes<D>() + 1024;
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attn_dq_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
               const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdo,
               const __grid_constant__ CUtensorMap mdq, BwdArgs a) {
    constexpr uint32_t kKeys = DqCfg<D>::kKeys, kVals = DqCfg<D>::kVals;
    constexpr int TB = tile_bytes<D>();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t q_full, do_full, s_full[2], dp_full, ds_full, all_done, k_full[kKeys], k_empty[kKeys],
        v_full[kVals], v_empty[kVals];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* abortp = &abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Geometry& g = a.g;

    // the longest rows first; the heads of a group next to one another, they read the same keys
    const int t = a.tiles - 1 - (int)(blockIdx.x / (unsigned)(g.n_seq * g.heads));
    const int nh = (int)(blockIdx.x % (unsigned)(g.n_seq * g.heads));
    const int n = nh / g.heads, h = nh - n * g.heads, hk = h / g.group;
    int lo, hi, from, to;
    live_range(g, n, lo, hi);
    key_tiles(g, t, lo, hi, from, to);
    const int steps = to - from;

    if (tid == 0) {
        mbar_init(&q_full, 1);
        mbar_init(&do_full, 1);
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        mbar_init(&dp_full, 1);
        mbar_init(&ds_full, 8);
        mbar_init(&all_done, 1);
        for (uint32_t s = 0; s < kKeys; ++s) {
            mbar_init(&k_full[s], 1);
            mbar_init(&k_empty[s], 1);
        }
        for (uint32_t s = 0; s < kVals; ++s) {
            mbar_init(&v_full[s], 1);
            mbar_init(&v_empty[s], 1);
        }
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
    // scores of even and odd steps, dP, dQ
    auto s_addr = [&](int i) { return tmem + (uint32_t)(i & 1) * 128u; };
    const uint32_t dp_t = tmem + 256u, dq_t = tmem + 384u;
    uint8_t* q_tile = smem;
    uint8_t* do_tile = smem + TB;
    auto k_tile = [&](uint32_t i) { return smem + (size_t)(2 + i % kKeys) * TB; };
    auto v_tile = [&](uint32_t i) { return smem + (size_t)(2 + kKeys + i % kVals) * TB; };

    if (warp == 8) {
        // ------------------------------------ copies ------------------------------------------------------
        if (lane == 0 && steps > 0) {
            mbar_arrive_expect_tx(&q_full, TB);
            load_tile<D>(q_tile, &mq, h, t * kTile, n, &q_full);
            mbar_arrive_expect_tx(&do_full, TB);
            load_tile<D>(do_tile, &mdo, h, t * kTile, n, &do_full);
            bool ok = true;
            uint32_t nkeys = 0, nvals = 0;
            // in the order of use: K_0 V_0 K_1 V_1 ...
            for (uint32_t i = 0; i < (uint32_t)steps && ok; ++i) {
                if (i >= kKeys && !mbar_wait_bounded(&k_empty[i % kKeys], ((i / kKeys) & 1u) ^ 1u, abortp)) {
                    ok = false;
                    break;
                }
                mbar_arrive_expect_tx(&k_full[i % kKeys], TB);
                load_tile<D>(k_tile(i), &mk, hk, (from + (int)i) * kTile, n, &k_full[i % kKeys]);
                ++nkeys;
                if (i >= kVals && !mbar_wait_bounded(&v_empty[i % kVals], ((i / kVals) & 1u) ^ 1u, abortp)) {
                    ok = false;
                    break;
                }
                mbar_arrive_expect_tx(&v_full[i % kVals], TB);
                load_tile<D>(v_tile(i), &mv, hk, (from + (int)i) * kTile, n, &v_full[i % kVals]);
                ++nvals;
            }
            if (!ok || *abortp) {  // gave up: let the copies land before the block's memory goes away
                auto land = [&](uint64_t* bar, uint32_t parity) {
                    const unsigned long long t0 = global_timer_ns();
                    while (!mbar_try_wait(bar, parity))
                        if (global_timer_ns() - t0 > kWaitLimitNs) break;
                };
                land(&q_full, 0);
                land(&do_full, 0);
                for (uint32_t i = nkeys > kKeys ? nkeys - kKeys : 0u; i < nkeys; ++i) land(&k_full[i % kKeys], (i / kKeys) & 1u);
                for (uint32_t i = nvals > kVals ? nvals - kVals : 0u; i < nvals; ++i) land(&v_full[i % kVals], (i / kVals) & 1u);
            }
        }
    } else if (warp == 9) {
        // ------------------------------------ products ----------------------------------------------------
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abortp));
            tc_fence_after();
            return ok;
        };
        auto scores = [&](uint32_t i) {
            if (!wait(&k_full[i % kKeys], (i / kKeys) & 1u)) return;
            zero_rows_outside<D>(k_tile(i), (from + (int)i) * kTile, lo, hi, lane);
            if (lane == 0) {
                mma_ss<D>(s_addr(i), smem_u32(q_tile), smem_u32(k_tile(i)));
                mma_commit(&s_full[i & 1]);
            }
        };
        auto dps = [&](uint32_t i) {
            if (!wait(&v_full[i % kVals], (i / kVals) & 1u)) return;
            zero_rows_outside<D>(v_tile(i), (from + (int)i) * kTile, lo, hi, lane);
            if (lane == 0) {
                mma_ss<D>(dp_t, smem_u32(do_tile), smem_u32(v_tile(i)));
                mma_commit(&dp_full);
                mma_commit(&v_empty[i % kVals]);
            }
        };
        if (steps > 0 && wait(&q_full, 0)) {
            scores(0);
            if (ok && wait(&do_full, 0)) dps(0);
            if (ok && steps > 1) scores(1);
            for (uint32_t i = 0; i < (uint32_t)steps && ok; ++i) {
                if (!wait(&ds_full, i & 1u)) break;
                if (lane == 0) {
                    const uint32_t kb = smem_u32(k_tile(i));
#pragma unroll
                    for (int ks = 0; ks < kTile / 16; ++ks)
                        mma_f16_ts(dq_t, s_addr(i) + (ks >> 2) * 64u + (ks & 3) * 8u, desc_mn(kb, ks), instr_desc(D, true), (i | ks) ? 1u : 0u);
                    mma_commit(&k_empty[i % kKeys]);
                }
                if (i + 1 < (uint32_t)steps) dps(i + 1);
                if (ok && i + 2 < (uint32_t)steps) scores(i + 2);
            }
        }
        __syncwarp();
        if (lane == 0) {
            mma_commit(&all_done);
            const unsigned long long t0 = global_timer_ns();
            while (!mbar_try_wait(&all_done, 0))
                if (global_timer_ns() - t0 > kWaitLimitNs) {
                    *abortp = 1;
                    break;
                }
        }
    } else {
        // ------------------------------------ probabilities, dS -------------------------------------------
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t mine = lanes + (uint32_t)half * 64u;
        const int pos = t * kTile + row;
        const bool live = pos >= lo && pos < hi;
        const int see = max(lo, pos - g.window + 1);
        const unsigned count = live ? (unsigned)(pos + 1 - see) : 0u;
        int full_from = 1 << 30, full_to = 0;  // key tiles that every row of the tile sees whole
        if (t * kTile >= lo && t * kTile + kTile <= hi) {
            full_from = (max(lo, t * kTile + kTile - g.window) + kTile - 1) / kTile;
            full_to = t;
        }
        const size_t at = (((size_t)n * g.heads + h) * a.tiles + t) * kTile + row;
        const float shift = a.shift[at], ndelta = a.ndelta[at];
        const float c = a.scale_log2;
        const uint64_t c2 = f32x2(c, c), shift2 = f32x2(shift, shift), ndelta2 = f32x2(ndelta, ndelta);
        bool ok = true;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abortp));
            tc_fence_after();
            return ok;
        };
        for (int i = 0; i < steps; ++i) {
            const int j = from + i;
            float p[64];
            if (!wait(&s_full[i & 1], (i >> 1) & 1)) break;
            {
                uint32_t s[2][32];
                tmem_ld32(s_addr(i) + mine, s[0]);
                tmem_ld32(s_addr(i) + mine + 32u, s[1]);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const uint32_t* x = &s[k >> 4][(k & 15) * 2];
                    f32x2_split(f32x2_fma(f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), c2, shift2), p[2 * k], p[2 * k + 1]);
                }
            }
#pragma unroll
            for (int k = 0; k < 64; ++k) p[k] = ex2_approx(p[k]);
            if (j < full_from || j >= full_to) {
                const int first = j * kTile + half * 64 - see;
#pragma unroll
                for (int k = 0; k < 64; ++k)
                    if ((unsigned)(first + k) >= count) p[k] = 0.f;
            }
            if (!wait(&dp_full, i & 1)) break;
            {
                uint32_t s[2][32], b[32];
                tmem_ld32(dp_t + mine, s[0]);
                tmem_ld32(dp_t + mine + 32u, s[1]);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const uint32_t* x = &s[k >> 4][(k & 15) * 2];
                    float e, f;
                    f32x2_split(f32x2_mul(f32x2(p[2 * k], p[2 * k + 1]), f32x2_add(f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), ndelta2)), e, f);
                    b[k] = pack_bf16x2(e, f);
                }
                tmem_st32(s_addr(i) + mine, b);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ds_full);
        }
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&all_done, 0, abortp));
        tc_fence_after();
        if (ok) {  // each half writes half of the columns
#pragma unroll 1
            for (int i = half * (D / 64); i < (half + 1) * (D / 64); ++i) {
                float f[32];
                if (steps > 0) {
                    uint32_t o[32];
                    tmem_ld32(dq_t + lanes + 32u * i, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = live ? __uint_as_float(o[k]) * a.scale : 0.f;
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) f[k] = 0.f;
                }
                stage_row32(q_tile, row, i, f);
            }
            fence_proxy_async_smem();
        }
        named_barrier(1, 256);
        if (tid == 0 && !*abortp) {
            store_tile<D>(&mdq, q_tile, g.head_dim, h, t * kTile, n);
            bulk_commit();
            bulk_wait_all<0>();
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

// ---- host -------------------------------------------------------------------------------------------------------

struct Maps {
    CUtensorMap q, k, v, dout, dq, dk, dv;
};

template <int D>
cudaError_t launch_bwd(const Maps& m, const BwdArgs& a, cudaStream_t st) {
    cudaError_t e = cudaFuncSetAttribute(attn_dkv_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DkvCfg<D>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_dq_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)DqCfg<D>::kSmem);
    if (e != cudaSuccess) return e;
    const unsigned nk = (unsigned)(a.g.n_seq * a.g.kv_heads), nh = (unsigned)(a.g.n_seq * a.g.heads);
    attn_dkv_kernel<D><<<nk * (unsigned)a.tiles, kThreads, DkvCfg<D>::kSmem, st>>>(m.q, m.k, m.v, m.dout, m.dk, m.dv, a);
    attn_dq_kernel<D><<<nh * (unsigned)a.tiles, kThreads, DqCfg<D>::kSmem, st>>>(m.q, m.k, m.v, m.dout, m.dq, a);
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
    return RAPID_OK;
}

size_t row_terms(const rapid_attn_desc_t& d) {  // floats of one of the two arrays
    return (size_t)((d.seq_len + kTile - 1) / kTile) * kTile * (size_t)d.n_seq * (size_t)d.n_heads;
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
    Maps m;
    if (!make_head_map(&m.q, q, d, d.n_heads, d.ld_q) || !make_head_map(&m.k, k, d, d.n_kv_heads, d.ld_k) ||
        !make_head_map(&m.v, v, d, d.n_kv_heads, d.ld_v) || !make_head_map(&m.dout, dout, d, d.n_heads, d.ld_dout) ||
        !make_head_map(&m.dq, dq, d, d.n_heads, d.ld_dq) || !make_head_map(&m.dk, dk, d, d.n_kv_heads, d.ld_dk) ||
        !make_head_map(&m.dv, dv, d, d.n_kv_heads, d.ld_dv))
        return RAPID_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (policy::clear_stats(stats, st) != cudaSuccess) return RAPID_ERR_CUDA;
    float* shift = static_cast<float*>(workspace);
    float* ndelta = shift + terms;
    BwdArgs a;
    a.g = make_geometry(d, bounds);
    a.scale = (float)d.scale;
    a.scale_log2 = (float)(d.scale * kLog2eD);
    a.tiles = (d.seq_len + kTile - 1) / kTile;
    a.shift = shift;
    a.ndelta = ndelta;
    a.stats = stats;
    int lanes_log2 = 0;
    while ((8 << lanes_log2) < d.head_dim) ++lanes_log2;
    const int64_t blocks = (((int64_t)terms << lanes_log2) + 255) / 256;
    if (blocks > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;
    attn_row_terms_kernel<<<(unsigned)blocks, 256, 0, st>>>(a.g, a.tiles, lanes_log2, static_cast<const uint16_t*>(out), d.ld_out,
                                                            static_cast<const uint16_t*>(dout), d.ld_dout, lse, shift, ndelta);
    const cudaError_t e = d.head_dim <= 64 ? launch_bwd<64>(m, a, st) : launch_bwd<128>(m, a, st);
    return e == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
