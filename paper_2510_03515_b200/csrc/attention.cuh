// What the attention kernels share: tiles, tensor-memory operands, geometry of the padded grid.
//
// Every operand tile is 128 positions of one head, [128][D] bf16 (D = 64 or 128; narrower heads are filled with zeros by
// the copy), in shared memory as D / 64 boxes of 128 rows x 128 bytes with the 128-byte swizzle.  Such a box serves as a
// K-major operand (contraction over the head's elements) and as an MN-major one (contraction over positions) alike, so
// nothing is ever transposed.  The tensor map has four dimensions (element, head, position, generation): a tile that
// reaches past the end of a generation reads zeros there and its stores are cut off.
//
// Positions outside a generation's bounds may hold anything.  They are masked out of the scores, and wherever such a
// row is summed over (0 x NaN is NaN), a warp overwrites it with zeros in shared memory before the product.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "policy_ops.cuh"
#include "tma_pipe.cuh"
#include "umma_gemm.cuh"

namespace rapid {
namespace attn {

using umma::tc_fence_after;
using umma::tc_fence_before;
using umma::tmem_alloc;
using umma::tmem_dealloc;
using umma::tmem_ld32;
using umma::tmem_ld_wait;
using umma::tmem_relinquish;

constexpr int kTile = 128;              // positions of a tile
constexpr int kBoxBytes = kTile * 128;  // one box: 128 rows of 64 elements

template <int D>
__host__ __device__ constexpr int tile_bytes() {
    return D / 64 * kBoxBytes;
}

// ---- PTX ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void tma_load_4d(void* smem_dst, const CUtensorMap* map, int x, int h, int t, int n, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], "
        "[%2];" ::"r"(smem_u32(smem_dst)),
        "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(h), "r"(t), "r"(n)
        : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, const void* smem_src, int x, int h, int t, int n) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(map),
                 "r"(smem_u32(smem_src)), "r"(x), "r"(h), "r"(t), "r"(n)
                 : "memory");
}
// True in one lane of a converged warp.  The whole loop that issues products runs inside `if (elect_one())`: the compiler
// then knows that one lane runs and keeps operands in uniform registers.  Measured for 128 x 64 x 16 (operands in tensor
// and shared memory): one product takes 33 cycles this way, 67 when the lane is chosen by a predicate.  Products are
// accepted only a few ahead, so what the lane does between two groups of them is time the tensor cores lose: a group of
// four with a wait before it and two commits after takes 326 cycles in one lane, 549 when the whole warp waits and votes.
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(e));
    return e != 0;
}

// A shared-memory descriptor as umma::smem_desc builds it, split in halves: the upper one is the same for every tile, and
// stepping through a tile is an addition to the lower one.
constexpr uint32_t kDescHi = 0x40004040u;  // stride offset 1024, version 1, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) { return (saddr >> 4) | ((lbo_bytes >> 4) << 16); }

// D[tmem] (+)= A[smem] * B[smem]
__device__ __forceinline__ void mma_ss_1(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 a, {%1, %5};\n\t"
        "mov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: lane i of A holds row i, a 32-bit column two consecutive bf16 along K
__device__ __forceinline__ void mma_ts_1(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi)
        : "memory");
}
using umma::mma_commit;  // arrive on a barrier once every product issued so far by this lane has ended

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- descriptors ------------------------------------------------------------------------------------------------

// As umma::instr_desc, for M = 128 and any N: f32 = bf16 x bf16, A K-major, B K-major or MN-major.
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}
// Lower descriptor halves of a tile: contraction over the head's elements (K-major; step `ks` of 16 elements), and over
// positions (MN-major; a step of 16 positions is 2048 bytes further on).
__device__ __forceinline__ uint32_t tile_k(uint32_t tile) { return desc_lo(tile, 16); }
__device__ __forceinline__ uint32_t tile_mn(uint32_t tile) { return desc_lo(tile, kBoxBytes); }
__device__ __forceinline__ constexpr uint32_t step_k(int ks) { return (uint32_t)((ks >> 2) * kBoxBytes + (ks & 3) * 32) >> 4; }
__device__ __forceinline__ constexpr uint32_t step_mn(int ks) { return (uint32_t)ks * 2048u >> 4; }

// D[128 x 128] = A[128 x D] * B[128 x D]^T, both tiles K-major in shared memory
template <int D>
__device__ __forceinline__ void mma_rows(uint32_t d_tmem, uint32_t a_tile, uint32_t b_tile) {
    const uint32_t a = tile_k(a_tile), b = tile_k(b_tile);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        mma_ss_1(d_tmem, a + step_k(ks), b + step_k(ks), instr_desc(kTile, false), ks > 0 ? 1u : 0u);
}

// acc[128 x D] (+)= M[128 x 128] * B[128 x D], M in tensor memory as bf16, 32 of its columns in 16 32-bit columns and the
// next 32 `stride` columns further on; B a tile used MN-major
template <int D>
__device__ __forceinline__ void mma_sum(uint32_t acc, uint32_t m, uint32_t stride, uint32_t b_tile, uint32_t more) {
    const uint32_t b = tile_mn(b_tile);
#pragma unroll
    for (int ks = 0; ks < kTile / 16; ++ks)
        mma_ts_1(acc, m + (ks >> 1) * stride + (ks & 1) * 8u, b + step_mn(ks), instr_desc(D, true), ks > 0 ? 1u : more);
}

template <int D>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, int h, int t0, int n, uint64_t* bar) {
#pragma unroll
    for (int b = 0; b < D / 64; ++b) tma_load_4d(dst + b * kBoxBytes, map, b * 64, h, t0, n, bar);
}
template <int D>
__device__ __forceinline__ void store_tile(const CUtensorMap* map, const uint8_t* src, int head_dim, int h, int t0, int n) {
#pragma unroll
    for (int b = 0; b < D / 64; ++b)
        if (b * 64 < head_dim) tma_store_4d(map, src + b * kBoxBytes, b * 64, h, t0, n);
}

// Wait for a phase of a barrier, bounded.  The first poll has no suspension hint: a phase that is over already then costs
// a few tens of cycles.
__device__ __forceinline__ bool wait_one(uint64_t* bar, uint32_t parity, volatile int* abortp) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done ? true : mbar_wait_bounded(bar, parity, abortp);
}
// The same for a whole warp; all lanes get the same answer.
__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abortp) {
    return __all_sync(0xffffffffu, wait_one(bar, parity, abortp));
}

// Place in a ring of `N` buffers: buffer number and the parity of its current use.
template <uint32_t N>
struct Place {
    uint32_t s = 0, parity = 0;
    __device__ __forceinline__ void step(uint32_t by = 1) {
        s += by;
        if (s >= N) {
            s -= N;
            parity ^= 1u;
        }
    }
};

// Tiles that hold dead rows ("dirty") come through a warp of their own: the copy reports to `raw`, the cleaning warp zeroes
// the dead rows and reports to the tile's ordinary barrier in the copy's place, and the readers notice nothing.
struct RawParity {
    uint32_t bits = 0;  // one for each buffer of a ring
    __device__ __forceinline__ uint32_t flip(uint32_t s) {  // parity of this use
        const uint32_t p = (bits >> s) & 1u;
        bits ^= 1u << s;
        return p;
    }
};

// After giving up: wait (again bounded) for something that is under way to arrive.
__device__ __forceinline__ void wait_landed(uint64_t* bar, uint32_t parity) {
    const unsigned long long t0 = global_timer_ns();
    while (!mbar_try_wait(bar, parity))
        if (global_timer_ns() - t0 > kWaitLimitNs) break;
}

// Wait for the commit of the last products, with the wait's own limit.
__device__ __forceinline__ void wait_drained(uint64_t* bar, volatile int* abortp) {
    const unsigned long long t0 = global_timer_ns();
    while (!mbar_try_wait(bar, 0))
        if (global_timer_ns() - t0 > kWaitLimitNs) {
            *abortp = 1;
            break;
        }
}

// ---- work handed out by the hardware ------------------------------------------------------------------------------
//
// A grid has one block for each piece of work, but a block that is done cancels the launch of a waiting one and does its
// work instead (clusterlaunchcontrol), until none is left.  Barriers, tensor memory and the copies' descriptors are set up
// once for each SM, the next piece's loads run under the end of this one, and the pieces still go to whoever is free.
// The copying lane asks, when it has issued the last loads of a piece (asking earlier would tie the next piece to a block
// that is still busy for long: dK, dV of 64 x 1024 took 410 us instead of 325), works out what the piece is and leaves it
// in shared memory for the other roles, which so never wait for the bounds to come from memory.
template <class W>  // the piece: plain data, a multiple of 16 bytes, with a member `end`: nothing is left
struct WorkQueue {
    static_assert(sizeof(W) % 16 == 0, "copied in 16-byte units");
    uint4 answer;
    W piece[2];
    uint64_t answered, full[2], empty[2];
};

template <class W>
__device__ __forceinline__ void work_init(WorkQueue<W>* q, uint32_t readers) {
    mbar_init(&q->answered, 1);
    for (int i = 0; i < 2; ++i) {
        mbar_init(&q->full[i], 1);
        mbar_init(&q->empty[i], readers);
    }
}
// Publish piece number k (0, 1, ...).  False: gave up.
template <class W>
__device__ __forceinline__ bool work_put(WorkQueue<W>* q, uint32_t k, const W& w, volatile int* abortp) {
    if (k >= 2 && !wait_one(&q->empty[k & 1u], ((k >> 1) & 1u) ^ 1u, abortp)) return false;
    q->piece[k & 1u] = w;
    mbar_arrive(&q->full[k & 1u]);
    return true;
}
// Ask for another block's work, for the k-th time; its number, -1 where there is none (then do not ask again), -2: gave up.
template <class W>
__device__ __forceinline__ int work_ask(WorkQueue<W>* q, uint32_t k, volatile int* abortp) {
    mbar_arrive_expect_tx(&q->answered, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                     smem_u32(&q->answer)),
                 "r"(smem_u32(&q->answered))
                 : "memory");
    if (!wait_one(&q->answered, k & 1u, abortp)) {
        wait_landed(&q->answered, k & 1u);  // it must not arrive in a block that has gone
        return -2;
    }
    uint32_t x, got;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
        "ld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.u32 %1, 1, 0, p;\n\t"
        "mov.u32 %0, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
        : "=r"(x), "=r"(got)
        : "r"(smem_u32(&q->answer))
        : "memory");
    fence_proxy_async_smem();  // the read comes before the next answer's write
    return got ? (int)x : -1;
}
// One lane takes piece k.  False when there is none (or the wait gave up).
template <class W>
__device__ __forceinline__ bool work_take_one(WorkQueue<W>* q, uint32_t k, W& w, volatile int* abortp) {
    if (!wait_one(&q->full[k & 1u], (k >> 1) & 1u, abortp)) return false;
    w = q->piece[k & 1u];
    mbar_arrive(&q->empty[k & 1u]);
    return !w.end;
}
// The same for a whole warp.
template <class W>
__device__ __forceinline__ bool work_take(WorkQueue<W>* q, uint32_t k, W& w, int lane, volatile int* abortp) {
    if (!wait_all(&q->full[k & 1u], (k >> 1) & 1u, abortp)) return false;
    w = q->piece[k & 1u];
    __syncwarp();
    if (lane == 0) mbar_arrive(&q->empty[k & 1u]);
    return !w.end;
}

// The largest of three (one instruction at the rate of the two-operand form).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// ---- results ------------------------------------------------------------------------------------------------------
//
// A thread holds (part of) a row; written straight to memory, every store of a warp would touch 32 lines, and the 32 KB of a
// tile kept the load/store unit busy for 2000 cycles.  Results go through shared memory and a tiled store instead; tiles
// without a live row, which are only zeros, are written directly.

// Row `row` of a tile in shared memory <- 32 values at columns [32 c, 32 c + 32), as bf16, in the layout of the copies.
__device__ __forceinline__ void stage_row32(uint8_t* tile, int row, int c, const float (&f)[32]) {
    uint8_t* box = tile + (c >> 1) * kBoxBytes;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<uint4*>(box + umma::swz128(row, (c & 1) * 4 + k)) =
            make_uint4(pack_bf16x2(f[8 * k], f[8 * k + 1]), pack_bf16x2(f[8 * k + 2], f[8 * k + 3]),
                       pack_bf16x2(f[8 * k + 4], f[8 * k + 5]), pack_bf16x2(f[8 * k + 6], f[8 * k + 7]));
}
// 32 accumulator columns of a row, times `factor`, to the same place (zeros where not `live`).
__device__ __forceinline__ void stage_acc32(uint8_t* tile, int row, int c, uint32_t taddr, bool live, float factor) {
    uint32_t o[32];
    tmem_ld32(taddr, o);
    tmem_ld_wait();
    float f[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) f[k] = live ? __uint_as_float(o[k]) * factor : 0.f;
    stage_row32(tile, row, c, f);
}
// Rows [t0, t0 + 128) of head h of generation n <- zeros, by `threads` threads; head_dim is a multiple of 8.
__device__ __forceinline__ void zero_tile(uint16_t* out, int64_t ld, int seq_len, int head_dim, int h, int t0, int n, int thread, int threads) {
    const int per_row = head_dim / 8;
    for (int i = thread; i < kTile * per_row; i += threads) {
        const int r = i / per_row, c = i - r * per_row;
        if (t0 + r < seq_len)
            *reinterpret_cast<uint4*>(out + ((int64_t)n * seq_len + t0 + r) * ld + h * head_dim + c * 8) = make_uint4(0, 0, 0, 0);
    }
}

// Roles of a block's warps: R warps hold rows, then one issues copies, one products, one clears dead rows, and one only gives up
// its registers.  The row warps take what the four others leave; the shares of a quarter of an SM add up to the launch's.
template <int R>
struct Roles {
    static constexpr int kRow = R, kCopy = R, kMma = R + 1, kClean = R + 2, kThreads = (R + 4) * 32;
    static __device__ __forceinline__ void take_registers() {
        if (R == 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");  // 2 x 208 + 88 = 3 x 168
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");         // 4 x 104 + 64 = 5 x 96
    }
    static __device__ __forceinline__ void leave_registers() {
        if (R == 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    }
    static_assert(R == 8 || R == 16, "the register shares above");
};

// ---- geometry -----------------------------------------------------------------------------------------------------

//
// Generations of at most half a tile share one: `parts` of them, `part` positions each, are a sequence of parts * part
// positions to everything that deals with tiles, and each row sees its own generation only.  (1335 x 40, 2 heads of 64: forward
// 40 us instead of 92; 4877 x 8, 9 heads of 128: 98 instead of 1042.)
struct Geometry {
    int n_seq, seq_len, heads, kv_heads, group, head_dim, window;  // window: a generation's length where there is none
    int part, parts;                                               // part = 0: generations have tiles of their own
    const int32_t* bounds;
};

// live positions [lo, hi) of generation n
__device__ __forceinline__ void live_range(const Geometry& g, int n, int& lo, int& hi) {
    lo = 0;
    hi = g.seq_len;
    if (g.bounds && g.part == 0) {
        lo = min(max(g.bounds[2 * n], 0), g.seq_len);
        hi = min(max(g.bounds[2 * n + 1], lo), g.seq_len);
    }
}

// The same for the generation that position `pos` of sequence n belongs to; lo, hi: what live_range said.
__device__ __forceinline__ void row_range(const Geometry& g, int n, int pos, int& lo, int& hi) {
    if (g.part == 0) return;
    const int gen = pos / g.part, start = gen * g.part;
    lo = hi = start;  // beyond the last one
    if (gen >= g.parts) return;
    hi += g.part;
    if (g.bounds) {
        const int32_t* b = g.bounds + 2 * ((size_t)n * g.parts + gen);
        lo = start + min(max(b[0], 0), g.part);
        hi = start + min(max(b[1], lo - start), g.part);
    }
}
// Where position pos < seq_len of sequence n has its lse.
__device__ __forceinline__ size_t lse_at(const Geometry& g, int n, int h, int pos) {
    if (g.part == 0) return ((size_t)n * g.heads + h) * g.seq_len + pos;
    const int gen = pos / g.part;
    return (((size_t)n * g.parts + gen) * g.heads + h) * g.part + (pos - gen * g.part);
}
template <bool SHARED>
__device__ __forceinline__ bool dirty(int tile, int lo, int hi) {
    return SHARED || tile * kTile < lo || tile * kTile + kTile > hi;
}
// Zero the dead rows of a tile, by one warp; the tile's first position is t0.
template <int D, bool SHARED>
__device__ __forceinline__ void zero_dead_rows(const Geometry& g, uint8_t* tile, int n, int t0, int lo, int hi, int lane) {
    if (!SHARED) {  // as below, the gradient of 3 x 4095 positions took 212 us instead of 194
        for (int i = lane; i < D / 64 * kTile * 8; i += 32) {
            const int row = (i >> 3) & (kTile - 1);
            if (t0 + row < lo || t0 + row >= hi) reinterpret_cast<uint4*>(tile)[i] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        __syncwarp();
        return;
    }
    uint32_t dead[kTile / 32];
#pragma unroll
    for (int k = 0; k < kTile / 32; ++k) {
        int a = lo, b = hi;
        row_range(g, n, t0 + 32 * k + lane, a, b);
        dead[k] = __ballot_sync(0xffffffffu, t0 + 32 * k + lane < a || t0 + 32 * k + lane >= b);
    }
#pragma unroll
    for (int box = 0; box < D / 64; ++box)
#pragma unroll
        for (int k = 0; k < kTile / 32; ++k)
            if (dead[k])
                for (int i = lane; i < 32 * 8; i += 32)
                    if ((dead[k] >> (i >> 3)) & 1u) reinterpret_cast<uint4*>(tile + box * kBoxBytes)[k * 256 + i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncwarp();
}

// First and one-past-last key tile that the live positions of query tile t see; empty where it has none.
__device__ __forceinline__ void key_tiles(const Geometry& g, int t, int lo, int hi, int& from, int& to) {
    const int first = max(t * kTile, lo), last = min(t * kTile + kTile, hi) - 1;
    from = to = 0;
    if (first > last) return;
    from = max(lo, first - g.window + 1) / kTile;
    to = last / kTile + 1;
}

// ---- host ---------------------------------------------------------------------------------------------------------

// Argument checks that both directions share, and the kernels' view of a descriptor.
rapid_status_t check_attn(const rapid_attn_desc_t* d);
Geometry make_geometry(const rapid_attn_desc_t& d, const int32_t* bounds);

// A call, or the part of one whose generations from `first` on are `d.n_seq` sequences of `parts` generations each.
struct Share {
    rapid_attn_desc_t d;  // n_seq, seq_len: of the sequences
    Geometry g;
    int64_t first_row;    // of the whole call's rows
};
// One share, or two where generations share tiles and the last sequence has fewer of them.
int make_shares(const rapid_attn_desc_t& d, const int32_t* bounds, Share (&shares)[2]);
inline const void* rows_from(const void* p, int64_t row, int64_t ld) { return static_cast<const uint16_t*>(p) + row * ld; }
inline void* rows_from(void* p, int64_t row, int64_t ld) { return static_cast<uint16_t*>(p) + row * ld; }

// Tensor map of [n_seq][seq_len][heads][head_dim] bf16 with row pitch `ld` elements, boxes of 128 positions x 64 elements.
bool make_head_map(CUtensorMap* map, const void* base, const rapid_attn_desc_t& d, int heads, int64_t ld);

}  // namespace attn
}  // namespace rapid
