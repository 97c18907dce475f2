// The rows of the losses of rapid_losses.h: every logit is read from memory once and its gradient written once, with the row held on
// one SM in between.  Three kernels, by the row's length: two rows by a warp, a row by a group of warps, and this one, a row by a block.
//
// Roles of a block of the longest rows: one producer warp draws rows from a counter and streams them into a ring of shared-memory
// stages with bulk copies; kWarps consumer warps read the stages; one warp gathers the chosen columns' logits ahead of time; one does
// what is done once a row: it joins the consumers' sums and computes the row's factor in double; one writes the zeros of the rows
// that do not count.
//
// A row's first reading takes its maximum and sum of exponentials chunk by chunk.  What fits stays: the first kKeep chunks in the
// consumers' registers, the last ones in their stages, so that the second reading, which writes the gradient, needs no memory
// traffic and hands its stages to the next row's loads as it goes.  Only of rows that are longer still are the chunks in between
// loaded again.
//
// Every wait on a barrier is bounded; a wait that gives up raises RAPID_ERR_TIMEOUT in the scratch and never traps.
//
// What bounds it: the bytes, at full length (8 x 1024 ragged rows of 151936 bf16: 633 us back to back, 0.99 of a copy's rate; with lists of
// 64 and a bucket 670, 0.93).  Where all rows count, the two sweeps do: an element costs two exponentials and some ten instructions
// (4096 rows of 151936: 449 us, 0.86).
#include <algorithm>
#include <type_traits>

#include "loss_rows.cuh"
#include "tma_pipe.cuh"

namespace rapid {
namespace losses {

namespace {

// Vector `at` of a row, from place `p`; columns behind the last one read as -inf.
template <int DT>
__device__ __forceinline__ uint4 edge_vector(const uint4* p, int at, int nvec, int rest) {
    using E = Elem<DT>;
    constexpr uint32_t kNone = DT == RAPID_BF16 ? 0xff80ff80u : 0xff800000u;
    uint4 v = make_uint4(kNone, kNone, kNone, kNone);
    if (at < nvec) v = *p;
    else if (at == nvec && rest) {
        const typename E::T* e = reinterpret_cast<const typename E::T*>(p);
        uint32_t w[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
        for (int i = 0; i < E::kPer; ++i) {
            if (i >= rest) continue;
            if constexpr (DT == RAPID_BF16) {
                const uint32_t b = e[i];
                w[i / 2] = (i & 1) ? ((w[i / 2] & 0xffffu) | (b << 16)) : ((w[i / 2] & 0xffff0000u) | b);
            } else {
                w[i] = __float_as_uint(e[i]);
            }
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}
// And its gradient, without the columns behind the last one.
template <int DT>
__device__ __forceinline__ void write_edge_vector(typename Elem<DT>::T* out, int at, const uint4& y, int nvec, int rest) {
    using E = Elem<DT>;
    if (at < nvec) st_stream(reinterpret_cast<uint4*>(out) + at, y);
    else if (at == nvec && rest) {
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < E::kPer; ++i) {
            if (i >= rest) continue;
            if constexpr (DT == RAPID_BF16) out[nvec * E::kPer + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            else out[nvec * E::kPer + i] = __uint_as_float(w[i]);
        }
    }
}

// ---- the longest rows ------------------------------------------------------------------------------------------

struct RingShape {
    int stages;   // of a chunk each
    int chunks;   // of a row
    int again;    // chunks of a row that are loaded a second time
    int list;     // chosen columns of a row, rounded up
    unsigned long long stride;
};

// Shared memory of one row's chosen columns: column, and logit or later value.
struct Slot {
    int* col;
    float* z;
};
constexpr int kSlotEntry = 8;  // bytes of one of them
// Without a gradient the clipped loss's rows are read by loss_tokens.cu.
template <class Op>
constexpr bool kAlwaysGrad = std::is_same<Op, ClipOp>::value;
// With the teacher's logits behind them, where there is a teacher (12 bytes for all would cost clip at 16384 bf16 one of its seven groups).
template <class Op>
constexpr int kSlotEntryT = std::is_same<Op, DistillOp>::value ? 12 : 8;
__device__ __forceinline__ Slot slot_at(uint8_t* base, int list) {
    float* p = reinterpret_cast<float*>(base);
    return Slot{reinterpret_cast<int*>(p), p + list};
}

// What the warps of a block tell each other, behind the stages in shared memory.
template <int kWarps>
struct Board {
    static constexpr int kStages = kWarps >= 16 ? 9 : 16;  // at most
    static constexpr int kQueue = kStages + 4;             // rows that are known to the block at a time, at most
    static constexpr int kZeros = 4;                       // rows that wait for their zeros
    static constexpr int kSlots = 3;                       // rows whose chosen columns are held
    uint64_t full[kStages], ready[kStages], empty[kStages], row[kQueue];
    uint64_t list[kSlots], value[kSlots], parts_in[2], grad[2], zero_full[kZeros], zero_empty[kZeros];
    long long row_q[kQueue], zero_q[kZeros];
    WarpPart parts[2][kWarps];
    GradConst grads[2];
    int abort_flag;
};

__device__ __forceinline__ void bulk_load_once(void* smem_dst, const void* gsrc, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(smem_u32(smem_dst)),
                 "l"(gsrc), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ uint64_t policy_first() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}

__device__ __forceinline__ uint64_t policy_normal() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}

// The next ticket.  (After atomicAdd() a warp waits for the result at once, some 1200 cycles.)
__device__ __forceinline__ unsigned int draw_ticket(const Scratch& w) {
    unsigned int t;
    asm volatile("atom.relaxed.gpu.global.add.u32 %0, [%1], 1;" : "=r"(t) : "l"(&w.head->ticket) : "memory");
    return t;
}

// By a whole warp; the lanes agree, so that all of them stay or all leave.
__device__ __noinline__ bool warp_wait_long(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag));
}
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return warp_wait_long(bar, parity, abort_flag);
}

// kWarps consumer warps, kVecs 16-byte vectors of a thread in a chunk, kKeep chunks in registers (0: without a gradient), kBlocks blocks on an SM
template <int DT, class Op, int kWarps, int kVecs, int kKeep, int kBlocks>
__global__ void __launch_bounds__((kWarps + 4) * 32, kBlocks) ring_kernel(RowsArgs a, Op op, RingShape sh) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int kLanes = kWarps * 32;          // consumer threads
    constexpr int kChunkVecs = kLanes * kVecs;   // vectors of a chunk
    constexpr int kChunk = kChunkVecs * 16;
    constexpr int kQueue = Board<kWarps>::kQueue, kZeros = Board<kWarps>::kZeros, kSlots = Board<kWarps>::kSlots;
    extern __shared__ __align__(128) uint8_t dyn[];
    uint8_t* ring = dyn;
    Board<kWarps>& bd = *reinterpret_cast<Board<kWarps>*>(dyn + (size_t)sh.stages * kChunk);
    uint8_t* slots = dyn + (size_t)sh.stages * kChunk + sizeof(Board<kWarps>);
    const int slot_bytes = sh.list * kSlotEntry;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int s = 0; s < sh.stages; ++s) {
            mbar_init(&bd.full[s], 1);
            mbar_init(&bd.ready[s], 1);
            mbar_init(&bd.empty[s], kWarps + (exclude(op) ? 1 : 0));  // the list's warp waits for the stages too
        }
        for (int q = 0; q < kQueue; ++q) mbar_init(&bd.row[q], 1);
        for (int q = 0; q < kZeros; ++q) {
            mbar_init(&bd.zero_full[q], 1);
            mbar_init(&bd.zero_empty[q], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bd.parts_in[s], kWarps);
            mbar_init(&bd.grad[s], 1);
        }
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(&bd.list[s], 1);
            mbar_init(&bd.value[s], 1);
        }
        bd.abort_flag = 0;
        mbar_init_fence();
    }
    __syncthreads();
    volatile int* abortp = &bd.abort_flag;

    constexpr bool grad = kKeep > 0;
    const int nvec = a.vocab / E::kPer, rest = a.vocab - nvec * E::kPer;
    constexpr int keep = kKeep;

    if (warp == kWarps) {
        // ------------------------------- producer -------------------------------------------
        const int all = nvec + (rest ? 1 : 0);  // vectors, inside the row: its pitch is a multiple of 16 bytes (which can be 4 GiB)
        const uint64_t first = policy_first(), normal = policy_normal();
        uint32_t it = 0, q = 0, zq = 0;
        bool ok = true;
        auto load = [&](const uint8_t* src, int c, bool more) {  // chunk c into the next stage; `more`: it will be read again
            const int s = it % sh.stages;
            const uint32_t use = it / sh.stages;
            if (use > 0 && !warp_wait(&bd.empty[s], (use & 1u) ^ 1u, abortp)) return false;
            if (lane == 0) {
                const int bytes = min(kChunkVecs, all - c * kChunkVecs) * 16;
                mbar_arrive_expect_tx(&bd.full[s], (uint32_t)bytes);
                bulk_load_once(ring + (size_t)s * kChunk, src + (size_t)c * kChunk, (uint32_t)bytes, &bd.full[s], more ? normal : first);
            }
            ++it;
            return true;
        };
        auto publish = [&](long long r) {
            if (lane == 0) {
                bd.row_q[q % kQueue] = r;
                mbar_arrive(&bd.row[q % kQueue]);
            }
            ++q;
        };
        auto zero = [&](long long r) {
            const uint32_t use = zq / kZeros;
            if (use > 0 && !warp_wait(&bd.zero_empty[zq % kZeros], (use & 1u) ^ 1u, abortp)) return false;
            if (lane == 0) {
                bd.zero_q[zq % kZeros] = r;
                mbar_arrive(&bd.zero_full[zq % kZeros]);
            }
            ++zq;
            return true;
        };
        while (ok) {
            unsigned int t = 0;
            if (lane == 0) t = draw_ticket(a.w);
            t = __shfl_sync(0xffffffffu, t, 0);
            if ((int64_t)t >= a.n_rows) break;
            const int64_t r = (int64_t)((unsigned long long)t * sh.stride % (unsigned long long)a.n_rows);
            if (a.w.state[r] != ROW_OK) {  // nobody reads this row
                if (grad) ok = zero(r);
                continue;
            }
            const uint8_t* src = static_cast<const uint8_t*>(a.logits) + (size_t)r * a.ld * sizeof(T);
            publish(r);
            for (int c = 0; c < sh.chunks && ok; ++c) ok = load(src, c, c >= keep && c < keep + sh.again);
            for (int c = keep; c < keep + sh.again && ok; ++c) ok = load(src, c, false);
        }
        if (ok) publish(-1);
        if (ok) zero(-1);
        __syncwarp();
        if (!ok || *abortp) {  // gave up: let the copies already issued land before the block's memory goes away
            const uint32_t from = it > (uint32_t)sh.stages ? it - sh.stages : 0u;
            for (uint32_t j = from; j < it; ++j) {
                const unsigned long long t0 = global_timer_ns();
                while (!mbar_try_wait(&bd.full[j % sh.stages], (j / sh.stages) & 1u))
                    if (global_timer_ns() - t0 > kWaitLimitNs) break;
            }
        }
    } else if (warp == kWarps + 2) {
        // ------------------------------- zeros for the rows that do not count ----------------
        for (uint32_t zq = 0;; ++zq) {
            if (!warp_wait(&bd.zero_full[zq % kZeros], (zq / kZeros) & 1u, abortp)) break;
            const int64_t r = bd.zero_q[zq % kZeros];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bd.zero_empty[zq % kZeros]);
            if (r < 0) break;
            T* out = static_cast<T*>(a.grad) + r * a.ld_grad;
#pragma unroll 4
            for (int v = lane; v < nvec; v += 32) st_stream(reinterpret_cast<uint4*>(out) + v, make_uint4(0, 0, 0, 0));
            if (lane < rest) out[nvec * E::kPer + lane] = E::put(0.f);
        }
    } else if (warp == kWarps + 3) {
        // ------------------------------- a row's chosen columns, ahead of the others --------
        const int n = list_size(op);
        const bool ex = exclude(op);
        int st = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (uint32_t jq = 0; ok; ++jq) {
            if (!warp_wait(&bd.row[jq % kQueue], (jq / kQueue) & 1u, abortp)) break;
            const int64_t r = bd.row_q[jq % kQueue];
            if (r < 0) break;
            const int s = jq % kSlots;
            // the row that had the slot, three ago, is done with: the values of the next one follow its sums, which the consumers give
            // when they have left the row before
            if (jq >= kSlots && !warp_wait(&bd.value[(jq - 2) % kSlots], (jq - 2) / kSlots & 1u, abortp)) break;
            const Slot slot = slot_at(slots + s * slot_bytes, sh.list);
            const T* row = static_cast<const T*>(a.logits) + r * a.ld;
            for (int j = lane; j < sh.list; j += 32) {
                const int v = j < n ? column(op, r, j) : -1;
                if (v >= 0) slot.z[j] = E::get(row[v]);
                slot.col[j] = v;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bd.list[s]);
            if (!ex) continue;
            // The list's columns are taken out of the sum; chunks loaded again come without: what is written for these columns is
            // written over.  Every stage is given back, those too: a wait for a stage's phase holds only until its next one.
            for (int c = 0; c < sh.chunks + sh.again; ++c) {
                if (!(ok = warp_wait(&bd.full[st], ph, abortp))) break;
                if (c < sh.chunks) {
                    T* e = reinterpret_cast<T*>(ring + (size_t)st * kChunk);
                    bool wrote = false;
                    for (int j = lane; j < sh.list; j += 32) {
                        const unsigned at = (unsigned)(slot.col[j] - c * kChunkVecs * E::kPer);
                        if (at < (unsigned)(kChunkVecs * E::kPer)) {
                            e[at] = E::put(-INFINITY);
                            wrote = true;
                        }
                    }
                    if (wrote) fence_proxy_async_smem();  // a bulk copy writes this stage next
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bd.ready[st]);
                }
                if (lane == 0) mbar_arrive(&bd.empty[st]);
                if (++st == sh.stages) {
                    st = 0;
                    ph ^= 1u;
                }
            }
        }
    } else if (warp == kWarps + 1) {
        // ------------------------------- once a row -----------------------------------------
        const double shared = shared_weight(op, rows_that_count(op_counts(op), op_blocks(op)));
        for (uint32_t jq = 0;; ++jq) {
            if (!warp_wait(&bd.row[jq % kQueue], (jq / kQueue) & 1u, abortp)) break;
            const int64_t r = bd.row_q[jq % kQueue];
            if (r < 0) break;
            const int s = jq & 1, slot_i = jq % kSlots;
            const uint32_t ph = (jq >> 1) & 1u;
            const Slot slot = slot_at(slots + slot_i * slot_bytes, sh.list);
            if (!warp_wait(&bd.list[slot_i], jq / kSlots & 1u, abortp)) break;
            auto mine = look<32>(op, head(op, r), shared, slot.col, slot.z, teacher(op, r));
            if (!warp_wait(&bd.parts_in[s], ph, abortp)) break;
            const RowStat st = join_parts(lane < kWarps ? bd.parts[s][lane] : WarpPart{0.0, -INFINITY, -INFINITY});
            const RowGrad g = finish(op, a, mine, st, slot.col, slot.z);
            if (lane == 0) {
                bd.grads[s] = grad_const<DT>(g, st.max, a.f);
                mbar_arrive(&bd.grad[s]);
            }
            values<32>(op, a, r, mine, g, st, slot.col, slot.z, teacher(op, r), true);
            __syncwarp();
            if (lane == 0) mbar_arrive(&bd.value[slot_i]);
        }
    } else {
        // ------------------------------- consumers ------------------------------------------
        const float off = shift_fraction(warp);
        const bool ex = exclude(op);
        const int whole = nvec / kChunkVecs;  // whole chunks of a row; at most one more
        int st = 0;
        uint32_t ph = 0, rph = 0;  // rph: a bit for each stage, as not every load into one is made ready
        auto next_stage = [&]() {
            if (++st == sh.stages) {
                st = 0;
                ph ^= 1u;
            }
        };
        auto give_back = [&](int s) {
            __syncwarp();
            if (lane == 0) mbar_arrive(&bd.empty[s]);
        };
        const uint4* my_ring = reinterpret_cast<const uint4*>(ring) + tid;
        auto read = [&](int s, uint4 (&v)[kVecs]) {
            const uint4* sv = my_ring + s * kChunkVecs;
#pragma unroll
            for (int j = 0; j < kVecs; ++j) v[j] = sv[j * kLanes];
        };
        auto read_edge = [&](const uint4* sv, int at) { return edge_vector<DT>(sv, at, nvec, rest); };
        for (uint32_t jq = 0;; ++jq) {
            if (!warp_wait(&bd.row[jq % kQueue], (jq / kQueue) & 1u, abortp)) break;
            const int64_t r = bd.row_q[jq % kQueue];
            if (r < 0) break;
            const int slot_i = jq & 1;  // of the sums and the factor
            const uint32_t sph = (jq >> 1) & 1u;
            const Slot slot = slot_at(slots + jq % kSlots * slot_bytes, sh.list);
            bool ok = true;
            uint4 kept[kKeep > 0 ? kKeep : 1][kVecs];
            int held = 0;  // stage of the first chunk that stays
            Part p;
            auto landed = [&]() {  // the next stage, for a first reading
                return ex ? warp_wait(&bd.ready[st], rph >> st & 1u, abortp) && ((rph ^= 1u << st), true) : warp_wait(&bd.full[st], ph, abortp);
            };
            const int held_from = grad ? keep + sh.again : sh.chunks;  // chunks from here on stay in their stages
            if (ok) {
                if (keep) {
#pragma unroll
                    for (int c = 0; c < kKeep; ++c)
                        if (ok && (ok = landed())) {
                            read(st, kept[c]);
                            p.template vectors<DT, kVecs>(kept[c], off, a.f);
                            give_back(st);
                            next_stage();
                        }
                }
                for (int c = keep; c < whole && ok; ++c) {
                    if (!(ok = landed())) break;
                    uint4 v[kVecs];
                    if (c == held_from) held = st;
                    read(st, v);
                    p.template vectors<DT, kVecs>(v, off, a.f);
                    if (c < held_from) give_back(st);
                    next_stage();
                }
                if (whole < sh.chunks && ok && (ok = landed())) {
                    if (whole == held_from) held = st;
#pragma unroll 1
                    for (int j = 0; j < kVecs; ++j) {
                        const int at = whole * kChunkVecs + j * kLanes + tid;
                        if (at - lane > nvec) break;  // nothing of this warp's any more
                        uint4 q[1] = {read_edge(my_ring + st * kChunkVecs + j * kLanes, at)};
                        p.template vectors<DT, 1>(q, off, a.f);
                    }
                    if (whole < held_from) give_back(st);
                    next_stage();
                }
                if (!ok) break;
                const WarpPart w = warp_part(p, a.f);
                // two rows ago's sums have been read
                if (!grad && jq >= 2 && !warp_wait(&bd.grad[slot_i], sph ^ 1u, abortp)) break;
                if (lane == 0) {
                    bd.parts[slot_i][warp] = w;
                    mbar_arrive(&bd.parts_in[slot_i]);
                }
            }
            if (!grad) continue;
            if (!warp_wait(&bd.grad[slot_i], sph, abortp)) break;
            // The row's constants stay in registers, but for lists with two blocks an SM, where there is none to spare: read for every chunk
            // (4096 distillation rows of 60000 bf16 242 -> 228 us; clip, which has some, 200 -> 205, and 4096 rows of 151936 472 -> 499).
            constexpr bool kAgain = kBlocks > 1 && !kAlwaysGrad<Op>;
            const Grad<DT> gr_kept(bd.grads[slot_i], a.f);
            auto row_grad = [&]() {
                if constexpr (kAgain) return Grad<DT>(bd.grads[slot_i], a.f);
                else return gr_kept;
            };
            T* out = static_cast<T*>(a.grad) + r * a.ld_grad;
            uint4* my_out = reinterpret_cast<uint4*>(out) + tid;
            // second reading: the gradient of a whole chunk
            auto write = [&](int c, const uint4 (&v)[kVecs]) {
                uint4* ov = my_out + c * kChunkVecs;
                const Grad<DT> gr = row_grad();
#pragma unroll
                for (int j = 0; j < kVecs; ++j) st_stream(ov + j * kLanes, gr.vector(v[j]));
            };
            // of a whole chunk c in stage s, which is then given back
            auto write_from = [&](int c, int s) {
                uint4 v[kVecs];
                read(s, v);
                write(c, v);
                give_back(s);
            };
            // and of the last chunk, where that is not whole
            auto write_edge = [&](int s) {
#pragma unroll 1
                for (int j = 0; j < kVecs; ++j) {
                    const int at = whole * kChunkVecs + j * kLanes + tid;
                    if (at - lane > nvec) break;
                    write_edge_vector<DT>(out, at, row_grad().vector(read_edge(my_ring + s * kChunkVecs + j * kLanes, at)), nvec, rest);
                }
                give_back(s);
            };
            for (int c = held_from; c < whole; ++c) {
                write_from(c, held);
                if (++held == sh.stages) held = 0;
            }
            if (whole < sh.chunks && whole >= held_from) write_edge(held);
            if (keep) {
#pragma unroll
                for (int c = 0; c < kKeep; ++c) write(c, kept[c]);
            }
            // chunks that are loaded again
            for (int c = keep; c < keep + sh.again && ok; ++c) {
                if (!(ok = warp_wait(&bd.full[st], ph, abortp))) break;
                if (c < whole) write_from(c, st);
                else write_edge(st);
                next_stage();
            }
            if (!ok) break;
            // the chosen columns over the vectors that hold them, which this warp wrote
            bool mine = false;
            for (int j = lane; j < sh.list; j += 32) mine |= slot.col[j] >= 0 && slot.col[j] / E::kPer % kLanes / 32 == warp;
            if (__any_sync(0xffffffffu, mine)) {
                if (!warp_wait(&bd.value[jq % kSlots], jq / kSlots & 1u, abortp)) break;
                __syncwarp();
                for (int j = lane; j < sh.list; j += 32) {
                    const int v = slot.col[j];
                    if (v >= 0 && v / E::kPer % kLanes / 32 == warp) out[v] = E::put(slot.z[j]);
                }
            }
        }
    }
    __syncthreads();
    if (tid == 0 && bd.abort_flag) {
        atomicMax(&a.w.head->status, (int)RAPID_ERR_TIMEOUT);
    }
    if (a.end.last_block) finish_rows(op, a, reinterpret_cast<double*>(dyn));
}

// ---- shorter rows ----------------------------------------------------------------------------------------------

// A group of G warps holds a whole row in its share of the SM's shared memory and does everything for it; as many groups as fit work
// side by side on an SM and hide one another's latencies.  A row comes in kParts bulk copies; the last warp to have read a part for the
// last time has the next row's part loaded in its place, so the warps meet only twice a row: to join their sums, and for the
// factor.  Rows are drawn from a counter, two ahead.  An element's instructions, and the two meetings, bound it: 32768 rows of 8192
// bf16 take 229 us (0.73 of a copy's rate), 16384 of 16384 209 (0.79), 8192 of 32000 221 (0.73), 8192 of 50000 306 (0.83).

constexpr int kParts = 2;

// Vectors of a thread at a time: eight hide more latency, where the registers are there for them (16384 rows of 16384 bf16 228 -> 220 us;
// eight warps a row 314 -> 325).
template <int G>
constexpr int kBatch = G < 8 ? 8 : 4;

struct GroupShape {
    int groups;          // of a block
    int row_bytes;       // place of a row
    int group_bytes;     // of a group in shared memory
    int part_vecs;       // vectors of a part, whole batches of every thread
    int parts;           // of a row
    int list;
};

struct GroupBoard {
    uint64_t full[kParts];
    WarpPart parts[2][8];
    GradConst grad;
    int read[kParts];    // warps that are through with a part
    long long next[2];   // the next row, ~row when it does not count; of odd and even turns
};

// The warps of a group together, with the OR of what they say: after a wait that gave up all leave together.
template <int G>
__device__ __forceinline__ bool group_sync(int id, bool flag) {
    uint32_t out;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %1, 0;\n\t"
        "barrier.cta.red.or.pred p, %2, %3, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(out)
        : "r"((uint32_t)flag), "r"(id), "n"(G * 32)
        : "memory");
    return out != 0;
}

template <int DT, class Op, int G>
__global__ void __launch_bounds__(512, 1) group_kernel(RowsArgs a, Op op, GroupShape sh) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int kLanes = G * 32;
    constexpr int U = kBatch<G>;  // vectors of a thread at a time
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ int abort_flag;
    __shared__ double weight;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / G, gw = warp % G, gt = threadIdx.x % kLanes;
    uint8_t* place = dyn + (size_t)group * sh.group_bytes;
    GroupBoard& bd = *reinterpret_cast<GroupBoard*>(place + sh.row_bytes);
    uint8_t* slots = place + sh.row_bytes + sizeof(GroupBoard);
    if (gt == 0) {
        for (int p = 0; p < kParts; ++p) {
            mbar_init(&bd.full[p], 1);
            bd.read[p] = 0;
        }
        mbar_init_fence();
    }
    if (threadIdx.x == 0) abort_flag = 0;
    volatile int* abortp = &abort_flag;
    const bool grad = kAlwaysGrad<Op> || a.grad != nullptr, ex = exclude(op);
    const int nvec = a.vocab / E::kPer, rest = a.vocab - nvec * E::kPer, all = nvec + (rest ? 1 : 0);
    const int n_list = list_size(op), id = group + 1;
    const unsigned int n_rows = (unsigned int)a.n_rows;
    const uint64_t once = policy_first();
    const float off = shift_fraction(gw);
    const uint4* row_place = reinterpret_cast<const uint4*>(place);

    uint32_t issued = 0, phase_of = 0;  // a bit for each part: loaded by this thread, and the phase of its last load
    auto load_part = [&](int64_t r, int p, uint32_t phase) {  // by one thread
        issued |= 1u << p;
        phase_of = (phase_of & ~(1u << p)) | phase << p;
        const int v = p * sh.part_vecs, bytes = min(sh.part_vecs, all - v) * 16;
        mbar_arrive_expect_tx(&bd.full[p], (uint32_t)bytes);
        bulk_load_once(place + (size_t)v * 16, static_cast<const uint8_t*>(a.logits) + (size_t)r * a.ld * sizeof(T) + (size_t)v * 16, (uint32_t)bytes,
                       &bd.full[p], once);
    };
    auto state_of = [&](unsigned int t) -> int { return t < n_rows ? (int)a.w.state[t] : ROW_MASKED; };

    // draws: the first ones are dealt out, one to every group of the grid; the group's first thread is ahead by two
    const unsigned int everyone = gridDim.x * sh.groups;
    unsigned int t0 = group * gridDim.x + blockIdx.x, t1 = 0, t2 = 0;
    int state1 = ROW_MASKED;
    int64_t row = t0 < n_rows ? (int64_t)t0 : a.n_rows;  // n_rows: there are none left
    bool live = state_of(t0) == ROW_OK;
    if (gt == 0) {
        t1 = everyone + draw_ticket(a.w);
        if (live)
            for (int p = 0; p < sh.parts; ++p) load_part(row, p, 0u);
    }
    if (warp == 0) {  // while the first rows come
        const double w = shared_weight(op, rows_that_count(op_counts(op), op_blocks(op)));
        if (lane == 0) weight = w;
    }
    __syncthreads();
    const double shared = weight;
    uint32_t ph = 0;         // phase of the parts, that is of the rows that are read
    int64_t pending = -1;    // the row whose chosen columns are still to be written
    bool ok = true;
    auto write_pending = [&]() {  // by the first warp, when the group has met since
        const Slot old = slot_at(slots + (ph ^ 1u) * sh.list * kSlotEntryT<Op>, sh.list);
        T* out = static_cast<T*>(a.grad) + pending * a.ld_grad;
#pragma unroll 1
        for (int j = lane; j < n_list; j += 32) {
            const int v = old.col[j];
            if (v >= 0) out[v] = E::put(old.z[j]);
        }
        pending = -1;
    };
    for (uint32_t turn = 0; row < a.n_rows; ++turn) {
        if (gt == 0) {
            t2 = draw_ticket(a.w);
            state1 = state_of(t1);
        }
        auto announce = [&]() {  // the next row, to the group
            if (gt == 0) {
                const int64_t r = t1 < n_rows ? (int64_t)t1 : a.n_rows;
                bd.next[turn & 1] = t1 < n_rows && state1 != ROW_OK ? ~r : r;
                t1 = everyone + t2;
            }
        };
        T* out = static_cast<T*>(a.grad) + row * a.ld_grad;
        if (!live) {
            if (grad) {
                for (int v = gt; v < nvec; v += kLanes) st_stream(reinterpret_cast<uint4*>(out) + v, make_uint4(0, 0, 0, 0));
                if (gt < rest) out[nvec * E::kPer + gt] = E::put(0.f);
            }
            announce();
            if (group_sync<G>(id, !ok)) break;
            __syncwarp();
            if (gw == 0 && pending >= 0) write_pending();
            const long long next = bd.next[turn & 1];
            row = next < 0 ? ~next : next;
            live = next >= 0 && next < a.n_rows;
            if (gt == 0 && live)
                for (int p = 0; p < sh.parts; ++p) load_part(row, p, ph);
            continue;
        }
        const Slot slot = slot_at(slots + ph * sh.list * kSlotEntryT<Op>, sh.list);
        if (gw == 0)
#pragma unroll 1
            for (int j = lane; j < n_list; j += 32) {
                const int v = column(op, row, j);
                if (teacher(op, row)) slot.z[sh.list + j] = teacher(op, row)[j];  // behind the slot's logits
                slot.col[j] = v;
            }
        const auto in = head(op, row);
        if (!grad) announce();
        auto read = [&](int at) { return edge_vector<DT>(row_place + at, at, nvec, rest); };
        long long next = 0;
        // this warp has read part p for the last time; the last one to say so has the next row's loaded there
        auto hand_over = [&](int p) {
            __syncwarp();
            if (lane != 0) return;
            __threadfence_block();
            if (atomicAdd(&bd.read[p], 1) != G - 1) return;
            __threadfence_block();
            bd.read[p] = 0;
            if (next >= 0 && next < a.n_rows) load_part(next, p, ph ^ 1u);
        };
        // ---- first reading ----
        if (!grad) {
            if (group_sync<G>(id, !ok)) break;  // the announcement
            __syncwarp();
            next = bd.next[turn & 1];
        }
        Part p;
        for (int q = 0; q < sh.parts && ok; ++q) {
            if (!(ok = warp_wait(&bd.full[q], ph, abortp))) break;
            const int from = q * sh.part_vecs, end = min(from + sh.part_vecs, all);
            if (ex) {  // the list's columns of this warp's vectors: their logits are noted and leave the sum
                bool wrote = false;
#pragma unroll 1
                for (int j = lane; j < n_list; j += 32) {
                    const int v = column(op, row, j), at = v / E::kPer;
                    if (v >= 0 && at >= from && at < end && (at - from) % kLanes / 32 == gw) {
                        T* e = reinterpret_cast<T*>(place) + v;
                        slot.z[j] = E::get(*e);
                        *e = E::put(-INFINITY);
                        wrote = true;
                    }
                }
                if (wrote) fence_proxy_async_smem();  // a bulk copy writes there next
                __syncwarp();
            } else if (!grad && gw == 0) {  // before the part goes
#pragma unroll 1
                for (int j = lane; j < n_list; j += 32) {
                    const int v = slot.col[j], at = v / E::kPer;
                    if (v >= 0 && at >= from && at < end) slot.z[j] = E::get(reinterpret_cast<const T*>(place)[v]);
                }
            }
            int v = from + gt;
            for (; v - lane + (U - 1) * kLanes + 31 < min(end, nvec); v += U * kLanes) {
                uint4 w[U];
#pragma unroll
                for (int j = 0; j < U; ++j) w[j] = row_place[v + j * kLanes];
                p.template vectors<DT, U>(w, off, a.f);
            }
#pragma unroll 1
            for (; v - lane < end; v += kLanes) {
                uint4 w[1] = {read(v)};
                p.template vectors<DT, 1>(w, off, a.f);
            }
            if (!grad) hand_over(q);
        }
        const WarpPart w = warp_part(p, a.f);
        RowStat st{0.0, 0.f};
        if (lane == 0) bd.parts[ph][gw] = w;
        if (group_sync<G>(id, !ok)) break;
        if (gw == 0) st = join_parts(lane < G ? bd.parts[ph][lane] : WarpPart{0.0, -INFINITY, -INFINITY});
        decltype(look<32>(op, in, shared, slot.col, slot.z, slot.z)) mine{};
        RowGrad g{0.0, 0.0};
        if (gw == 0) {
            if (!ex && grad)
#pragma unroll 1
                for (int j = lane; j < n_list; j += 32) {
                    const int v = slot.col[j];
                    if (v >= 0) slot.z[j] = E::get(reinterpret_cast<const T*>(place)[v]);
                }
            __syncwarp();
            mine = look<32>(op, in, shared, slot.col, slot.z, slot.z + sh.list);
            g = finish(op, a, mine, st, slot.col, slot.z);
            if (lane == 0) bd.grad = grad_const<DT>(g, st.max, a.f);
            if (grad) announce();
        }
        if (grad) {
            // ---- second reading ----
            if (group_sync<G>(id, !ok)) break;
            __syncwarp();
            next = bd.next[turn & 1];
            if (gw == 0 && pending >= 0) write_pending();
            const Grad<DT> gr(bd.grad, a.f);
            uint4* ov = reinterpret_cast<uint4*>(out);
            for (int q = 0; q < sh.parts; ++q) {
                const int from = q * sh.part_vecs, end = min(from + sh.part_vecs, all);
                int v = from + gt;
                for (; v - lane + (U - 1) * kLanes + 31 < min(end, nvec); v += U * kLanes) {
                    uint4 w[U];
#pragma unroll
                    for (int j = 0; j < U; ++j) w[j] = row_place[v + j * kLanes];
#pragma unroll
                    for (int j = 0; j < U; ++j) st_stream(ov + v + j * kLanes, gr.vector(w[j]));
                }
#pragma unroll 1
                for (; v - lane < end; v += kLanes) write_edge_vector<DT>(out, v, gr.vector(read(v)), nvec, rest);
                hand_over(q);
            }
        }
        if (gw == 0) {
            values<32>(op, a, row, mine, g, st, slot.col, slot.z, slot.z + sh.list, true);
            __syncwarp();
            if (grad) pending = row;
        }
        ph ^= 1u;
        row = next < 0 ? ~next : next;
        live = next >= 0 && next < a.n_rows;
    }
    if (grad && !group_sync<G>(id, *abortp != 0)) {
        __syncwarp();
        if (gw == 0 && pending >= 0) write_pending();
    }
    if (lane == 0 && *abortp) {  // gave up: let the copies already issued land before the block's memory goes away
        for (int p = 0; p < sh.parts; ++p) {
            const unsigned long long t = global_timer_ns();
            while ((issued >> p & 1u) && !mbar_try_wait(&bd.full[p], phase_of >> p & 1u))
                if (global_timer_ns() - t > kWaitLimitNs) break;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag) {
        atomicMax(&a.w.head->status, (int)RAPID_ERR_TIMEOUT);
    }
    if (a.end.last_block) finish_rows(op, a, reinterpret_cast<double*>(dyn));
}

// ---- the shortest rows ------------------------------------------------------------------------------------------

// Up to 8 KB a warp holds two rows at a time: it reads them one after the other, then does what is done once a row for both of them
// at once, half a warp each, and writes them one after the other.  That arithmetic, one value a row in double, is a chain of some
// thousands of cycles in which a warp that holds one row does nothing else: when 65536 rows of 4096 bf16 with 8 entries took 240 us so,
// they took 300 with one row a warp, and 297 with four, which leave six warps an SM.  Now 211; floor 146.
constexpr int kTogether = 2;

struct ShortShape {
    int warps;       // of a block
    int row_bytes;   // place of a row
    int warp_bytes;  // of a warp in shared memory
    int list;
    int slot_bytes;  // of a row's chosen columns
};

__device__ __forceinline__ void copy_word(void* smem_dst, const void* gsrc) {  // comes on its own
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(smem_dst)), "l"(gsrc) : "memory");
}
// What is known of a row's chosen columns ahead of time, into its slot, by one warp.
__device__ __forceinline__ void copy_list(const ClipOp& op, int64_t r, const Slot& slot, int) {
    if ((threadIdx.x & 31) == 0) copy_word(slot.col, op.targets + r);
}
__device__ __forceinline__ void copy_list(const DistillOp& op, int64_t r, const Slot& slot, int list) {
    for (int j = threadIdx.x & 31; j < op.k; j += 32) {
        copy_word(slot.col + j, op.index + r * op.ld + j);
        copy_word(slot.z + list + j, op.logit + r * op.ld + j);
    }
}

struct ShortBoard {
    uint64_t full[kTogether];
    WarpPart parts[kTogether];
    GradConst grads[kTogether];
};

template <int DT, class Op>
__global__ void __launch_bounds__(512, 1) short_kernel(RowsArgs a, Op op, ShortShape sh) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int U = 4, W = 32 / kTogether;
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ int abort_flag;
    __shared__ double weight;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t* place = dyn + (size_t)warp * sh.warp_bytes;
    ShortBoard& bd = *reinterpret_cast<ShortBoard*>(place + kTogether * sh.row_bytes);
    uint8_t* slots = place + kTogether * sh.row_bytes + sizeof(ShortBoard);
    if (lane == 0) {
        for (int k = 0; k < kTogether; ++k) mbar_init(&bd.full[k], 1);
        mbar_init_fence();
    }
    if (threadIdx.x == 0) abort_flag = 0;
    if (warp == 0) {
        const double w = shared_weight(op, rows_that_count(op_counts(op), op_blocks(op)));
        if (lane == 0) weight = w;
    }
    __syncthreads();
    volatile int* abortp = &abort_flag;
    const double shared = weight;
    const bool grad = kAlwaysGrad<Op> || a.grad != nullptr, ex = exclude(op);
    const int nvec = a.vocab / E::kPer, rest = a.vocab - nvec * E::kPer, all = nvec + (rest ? 1 : 0);
    const int n_list = list_size(op);
    const unsigned int n_rows = (unsigned int)a.n_rows, n_sets = (n_rows + kTogether - 1) / kTogether;
    const uint64_t once = policy_first();
    const float off = shift_fraction(0);

    uint32_t issued = 0, phase_of = 0;  // a bit for each place: loaded by this lane, and the phase of its last load
    uint32_t ph = 0;                    // phase of each place's next load, a bit each
    auto load_row = [&](unsigned int r, int k) {  // by one lane, into place k
        issued |= 1u << k;
        phase_of = (phase_of & ~(1u << k)) | (ph & 1u << k);
        mbar_arrive_expect_tx(&bd.full[k], (uint32_t)all * 16u);
        bulk_load_once(place + (size_t)k * sh.row_bytes, static_cast<const uint8_t*>(a.logits) + (size_t)r * a.ld * sizeof(T), (uint32_t)all * 16u,
                       &bd.full[k], once);
    };
    auto state_of = [&](unsigned int set) -> int {  // of the set's row that is this lane's
        const unsigned int r = set * kTogether + lane;
        return lane < kTogether && set < n_sets && r < n_rows ? (int)a.w.state[r] : ROW_MASKED;
    };
    auto slot_of = [&](uint32_t turn, int k) { return slot_at(slots + ((turn & 1u) * kTogether + k) * sh.slot_bytes, sh.list); };
    auto my_row = [&](unsigned int set) { return (int64_t)min(set * kTogether + lane / W, n_rows - 1); };
    auto copy_lists = [&](unsigned int set, uint32_t live, uint32_t turn) {
        for (int k = 0; k < kTogether; ++k)
            if (live >> k & 1u) copy_list(op, set * kTogether + k, slot_of(turn, k), sh.list);
    };
    // Sets are dealt out first, one to every warp of the grid, then drawn.  A load that is issued behind a row's stores comes back when
    // those have left the SM, thousands of cycles later; so what is needed of the next set is asked for before this one's are written.
    const unsigned int everyone = gridDim.x * sh.warps;
    unsigned int set = warp * gridDim.x + blockIdx.x, next = 0, draw = 0;
    if (lane == 0) {
        next = draw_ticket(a.w);
        draw = draw_ticket(a.w);
    }
    next = everyone + __shfl_sync(0xffffffffu, next, 0);
    uint32_t live = __ballot_sync(0xffffffffu, state_of(set) == ROW_OK);
    int state = state_of(next);
    for (int k = 0; k < kTogether; ++k)
        if (lane == 0 && (live >> k & 1u)) load_row(set * kTogether + k, k);
    copy_lists(set, live, 0u);
    auto in = head(op, my_row(set));
    bool ok = true;
    for (uint32_t turn = 0; set < n_sets && ok; ++turn) {
        const unsigned int row0 = set * kTogether, later = everyone + __shfl_sync(0xffffffffu, draw, 0);
        if (lane == 0) draw = draw_ticket(a.w);
        const uint32_t live_next = __ballot_sync(0xffffffffu, state == ROW_OK);
        asm volatile("cp.async.wait_all;" ::: "memory");  // this set's columns
        if (grad)
            for (int k = 0; k < kTogether; ++k)
                if (!(live >> k & 1u) && row0 + k < n_rows) {  // nobody reads this row
                    T* out = static_cast<T*>(a.grad) + (int64_t)(row0 + k) * a.ld_grad;
                    for (int v = lane; v < nvec; v += 32) st_stream(reinterpret_cast<uint4*>(out) + v, make_uint4(0, 0, 0, 0));
                    if (lane < rest) out[nvec * E::kPer + lane] = E::put(0.f);
                }
        __syncwarp();
        auto read = [&](const uint4* p, int at) { return edge_vector<DT>(p + at, at, nvec, rest); };
        auto hand_over = [&](int k) {  // place k has been read for the last time
            __syncwarp();
            if (lane == 0 && (live_next >> k & 1u)) load_row(next * kTogether + k, k);
        };
        // ---- first reading ----
#pragma unroll 1
        for (int k = 0; k < kTogether && ok; ++k) {
            if (!(live >> k & 1u)) continue;
            if (!(ok = warp_wait(&bd.full[k], ph >> k & 1u, abortp))) break;
            ph ^= 1u << k;
            uint8_t* row = place + (size_t)k * sh.row_bytes;
            const uint4* p = reinterpret_cast<const uint4*>(row);
            const Slot slot = slot_of(turn, k);
            bool wrote = false;
#pragma unroll 1
            for (int j = lane; j < n_list; j += 32) {
                const int v = slot.col[j];
                if (v < 0) continue;
                T* e = reinterpret_cast<T*>(row) + v;
                slot.z[j] = E::get(*e);
                if (ex) *e = E::put(-INFINITY);  // left out of the sum
                wrote = ex;
            }
            if (wrote) fence_proxy_async_smem();  // a bulk copy writes there next
            __syncwarp();
            Part part;
            int v = lane;
            for (; v - lane + (U - 1) * 32 + 31 < nvec; v += U * 32) {
                uint4 q[U];
#pragma unroll
                for (int j = 0; j < U; ++j) q[j] = p[v + j * 32];
                part.template vectors<DT, U>(q, off, a.f);
            }
#pragma unroll 1
            for (; v - lane < all; v += 32) {
                uint4 q[1] = {read(p, v)};
                part.template vectors<DT, 1>(q, off, a.f);
            }
            const WarpPart w = warp_part(part, a.f);
            if (lane == 0) bd.parts[k] = w;
            if (!grad) hand_over(k);
        }
        if (!ok) break;
        __syncwarp();
        // ---- once a row, for all of them ----
        {
            const int k = lane / W;
            const bool mine = live >> k & 1u;
            const Slot slot = slot_of(turn, k);
            const RowStat st = one_part(mine ? bd.parts[k] : WarpPart{0.0, -INFINITY, -INFINITY});
            auto row = look<W>(op, in, shared, slot.col, slot.z, slot.z + sh.list);
            const RowGrad g = finish(op, a, row, st, slot.col, slot.z);
            if (lane % W == 0) bd.grads[k] = grad_const<DT>(g, st.max, a.f);
            values<W>(op, a, my_row(set), row, g, st, slot.col, slot.z, slot.z + sh.list, mine);
        }
        __syncwarp();
        copy_lists(next, live_next, turn + 1);
        in = head(op, my_row(next));
        state = state_of(later);
        // ---- second reading ----
        if (grad) {
#pragma unroll 1
            for (int k = 0; k < kTogether; ++k) {
                if (!(live >> k & 1u)) {
                    hand_over(k);
                    continue;
                }
                const uint4* p = reinterpret_cast<const uint4*>(place + (size_t)k * sh.row_bytes);
                const Slot slot = slot_of(turn, k);
                const Grad<DT> gr(bd.grads[k], a.f);
                T* out = static_cast<T*>(a.grad) + (int64_t)(row0 + k) * a.ld_grad;
                uint4* ov = reinterpret_cast<uint4*>(out);
                int v = lane;
                for (; v - lane + (U - 1) * 32 + 31 < nvec; v += U * 32) {
                    uint4 q[U];
#pragma unroll
                    for (int j = 0; j < U; ++j) q[j] = p[v + j * 32];
#pragma unroll
                    for (int j = 0; j < U; ++j) st_stream(ov + v + j * 32, gr.vector(q[j]));
                }
#pragma unroll 1
                for (; v - lane < all; v += 32) write_edge_vector<DT>(out, v, gr.vector(read(p, v)), nvec, rest);
                hand_over(k);
#pragma unroll 1
                for (int j = lane; j < n_list; j += 32) {  // the chosen columns over the vectors
                    const int c = slot.col[j];
                    if (c >= 0) out[c] = E::put(slot.z[j]);
                }
            }
        } else {
            for (int k = 0; k < kTogether; ++k)
                if (!(live >> k & 1u)) hand_over(k);
        }
        __syncwarp();  // the slots have been read
        set = next;
        next = later;
        live = live_next;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0 && *abortp) {  // gave up: let the copies already issued land before the block's memory goes away
        for (int k = 0; k < kTogether; ++k) {
            const unsigned long long t = global_timer_ns();
            while ((issued >> k & 1u) && !mbar_try_wait(&bd.full[k], phase_of >> k & 1u))
                if (global_timer_ns() - t > kWaitLimitNs) break;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag) atomicMax(&a.w.head->status, (int)RAPID_ERR_TIMEOUT);
    if (a.end.last_block) finish_rows(op, a, reinterpret_cast<double*>(dyn));
}

template <class Op>
cudaError_t launch(const RowsArgs& a, const Op& op, int list, int sm_count, cudaStream_t stream) {
    const size_t es = elem_size(a.dtype);
    const int64_t row_bytes = ((int64_t)a.vocab * es + 15) / 16 * 16;
    auto go = [&](auto kern, int warps, int vecs, int keep, int blocks, size_t board, int most) -> cudaError_t {
        RingShape sh{};
        const int chunk = warps * 32 * vecs * 16;
        sh.list = (list + 3) / 4 * 4;
        const size_t extra = board + 3 * (size_t)sh.list * kSlotEntry;
        // 228 KB an SM, of which 1 KB for each block is the system's; 227 KB a block
        const size_t room = std::min((size_t)227 * 1024, (size_t)228 * 1024 / blocks - 1024) - extra;
        sh.stages = std::min((int)(room / chunk), most);
        sh.chunks = (int)((row_bytes + chunk - 1) / chunk);
        sh.again = a.grad && sh.chunks > keep + sh.stages ? sh.chunks - keep - sh.stages : 0;
        const size_t smem = (size_t)sh.stages * chunk + extra;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        int64_t grid = (int64_t)sm_count * blocks;
        if (grid > a.n_rows) grid = a.n_rows;
        sh.stride = scatter_stride(a.n_rows);
        kern<<<(unsigned)grid, (warps + 4) * 32, smem, stream>>>(a, op, sh);
        return cudaGetLastError();
    };
    auto go_groups = [&](auto kern, int G, int batch) -> cudaError_t {
        GroupShape sh{};
        const int lanes = G * 32, all = (int)(row_bytes / 16);
        sh.list = (list + 3) / 4 * 4;
        // a row in two parts, so that the next row's first half comes while the second is read
        const int unit = lanes * batch;
        sh.part_vecs = ((all + kParts - 1) / kParts + unit - 1) / unit * unit;
        sh.parts = (all + sh.part_vecs - 1) / sh.part_vecs;
        sh.row_bytes = (int)row_bytes;
        sh.group_bytes = (int)((row_bytes + sizeof(GroupBoard) + 2 * sh.list * kSlotEntryT<Op> + 127) / 128 * 128);
        sh.groups = std::min((227 * 1024 - 128) / sh.group_bytes, 16 / G);
        const size_t smem = std::max((size_t)sh.groups * sh.group_bytes, kEndBytes);
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        const int64_t grid = std::min((int64_t)sm_count, a.n_rows);
        kern<<<(unsigned)grid, sh.groups * lanes, smem, stream>>>(a, op, sh);
        return cudaGetLastError();
    };
    auto go_short = [&](auto kern) -> cudaError_t {
        ShortShape sh{};
        sh.list = (list + 3) / 4 * 4;
        sh.row_bytes = (int)row_bytes;
        sh.slot_bytes = sh.list * kSlotEntryT<Op>;
        sh.warp_bytes = (int)((kTogether * row_bytes + sizeof(ShortBoard) + 2 * kTogether * sh.slot_bytes + 127) / 128 * 128);
        sh.warps = std::min((227 * 1024 - 128) / sh.warp_bytes, 16);
        const size_t smem = std::max((size_t)sh.warps * sh.warp_bytes, kEndBytes);
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        const int64_t sets = (a.n_rows + kTogether - 1) / kTogether;
        kern<<<(unsigned)std::min((int64_t)sm_count, sets), sh.warps * 32, smem, stream>>>(a, op, sh);
        return cudaGetLastError();
    };
    auto by_type = [&](auto dt) -> cudaError_t {
        constexpr int DT = decltype(dt)::value;
        // warps for a row: as many as leave at least two groups an SM and each thread two batches (16384 x 8192 bf16 in ones 285 us, in twos
        // 246; 8192 x 32000 in fours 229, in eights 249)
        // Few rows: as many warps for each as there are for all at once, 16 an SM (256 rows of 1000 bf16 21 -> 16 us, 512 of 4096 25 -> 18,
        // 1024 of 4096 28 -> 21, 64 of 32000 21 -> 19; where the rows do not fit side by side it makes no difference).
        const int64_t rows_sm = (a.n_rows + sm_count - 1) / sm_count;
        if (row_bytes <= 110 * 1024 && rows_sm <= 2) return go_groups(group_kernel<DT, Op, 8>, 8, kBatch<8>);
        if (row_bytes <= 55 * 1024 && rows_sm <= 4) return go_groups(group_kernel<DT, Op, 4>, 4, kBatch<4>);
        if (row_bytes <= 27 * 1024 && rows_sm <= 8) return go_groups(group_kernel<DT, Op, 2>, 2, kBatch<2>);
        if (row_bytes <= 8192) return go_short(short_kernel<DT, Op>);
        if (row_bytes <= 32768) return go_groups(group_kernel<DT, Op, 2>, 2, kBatch<2>);
        if (row_bytes <= 73728) return go_groups(group_kernel<DT, Op, 4>, 4, kBatch<4>);
        if (row_bytes <= 110 * 1024) return go_groups(group_kernel<DT, Op, 8>, 8, kBatch<8>);
        constexpr size_t b16 = sizeof(Board<16>);
        const bool grad = kAlwaysGrad<Op> || a.grad;
        if (grad && row_bytes <= 172 * 1024) return go(ring_kernel<DT, Op, 8, 4, 2, 2>, 8, 4, 2, 2, sizeof(Board<8>), Board<8>::kStages);
        // Lists need room beside the stages: chunks of 24 KB leave it, seven of 32 KB do not (16 x 512 rows of 151936 with 128 entries 844 us,
        // with a chunk that has to be loaded again 1174); without lists 32 KB cost a little less (4096 rows: 462, 469).
        constexpr int kV = std::is_same<Op, DistillOp>::value ? 3 : 4, kK = 7 - kV;
        if (grad) return go(ring_kernel<DT, Op, 16, kV, kK, 1>, 16, kV, kK, 1, b16, Board<16>::kStages);
        if constexpr (!kAlwaysGrad<Op>) return go(ring_kernel<DT, Op, 16, 4, 0, 1>, 16, 4, 0, 1, b16, Board<16>::kStages);
        return cudaErrorInvalidValue;
    };
    return a.dtype == RAPID_BF16 ? by_type(std::integral_constant<int, RAPID_BF16>{}) : by_type(std::integral_constant<int, RAPID_F32>{});
}

}  // namespace

cudaError_t launch_rows(const RowsArgs& a, const ClipOp& op, int sm_count, cudaStream_t stream) { return launch(a, op, 1, sm_count, stream); }
cudaError_t launch_rows(const RowsArgs& a, const DistillOp& op, int sm_count, cudaStream_t stream) {
    return launch(a, op, op.k, sm_count, stream);
}

}  // namespace losses
}  // namespace rapid
