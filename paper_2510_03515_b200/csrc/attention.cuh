// What the attention kernels share: tiles, tensor-memory operands, geometry of the padded grid.
//
// Every operand tile is 128 positions of one head, [128][D] bf16 (D = 64 or 128; narrower heads are filled with zeros by
// the copy), in shared memory as D / 64 boxes of 128 rows x 128 bytes with the 128-byte swizzle.  Such a box serves as a
// K-major operand (contraction over the head's elements) and as an MN-major one (contraction over positions) alike, so
// nothing is ever transposed.  The tensor map has four dimensions (element, head, position, generation): a tile that
// reaches past the end of a generation reads zeros there and its stores are cut off.
//
// Positions outside a generation's bounds may hold anything.  They are masked out of the scores, and wherever such a
// row is summed over (0 x NaN is NaN), the issuing warp overwrites it with zeros in shared memory before the product.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "policy_ops.cuh"
#include "tma_pipe.cuh"
#include "umma_gemm.cuh"

namespace rapid {
namespace attn {

using umma::mma_commit;
using umma::mma_f16;
using umma::smem_desc;
using umma::swz128;
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
// D[tmem] (+)= A[tmem] * B[smem]: lane i of A holds row i, a 32-bit column two consecutive bf16 along K
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
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
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// barrier of `count` threads of the block (id 1 .. 15; whole warps)
__device__ __forceinline__ void named_barrier(int id, int count) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(count) : "memory");
}

// ---- descriptors ------------------------------------------------------------------------------------------------

// As umma::instr_desc, for M = 128 and any N: f32 = bf16 x bf16, A K-major, B K-major or MN-major.
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}
// Step `ks` of 16 elements along the head: the K-major form of a tile.
__device__ __forceinline__ uint64_t desc_k(uint32_t tile, int ks) {
    return smem_desc(tile + (uint32_t)(ks >> 2) * kBoxBytes + (uint32_t)(ks & 3) * 32u, 16);
}
// Step `ks` of 16 positions: the MN-major form (the head's elements are the other dimension).
__device__ __forceinline__ uint64_t desc_mn(uint32_t tile, int ks) { return smem_desc(tile + (uint32_t)ks * 2048u, kBoxBytes); }

// D[128 x 128] = A[128 x D] * B[128 x D]^T, both tiles K-major in shared memory
template <int D>
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_tile, uint32_t b_tile) {
    constexpr uint32_t idesc = instr_desc(kTile, false);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) mma_f16(d_tmem, desc_k(a_tile, ks), desc_k(b_tile, ks), idesc, ks > 0 ? 1u : 0u);
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

// One warp overwrites with zeros the rows of a tile that lie outside [lo, hi), before a product reads them.
template <int D>
__device__ __forceinline__ void zero_rows_outside(uint8_t* tile, int t0, int lo, int hi, int lane) {
    if (t0 >= lo && t0 + kTile <= hi) return;
    for (int i = lane; i < D / 64 * kTile * 8; i += 32) {
        const int row = (i >> 3) & (kTile - 1);
        if (t0 + row < lo || t0 + row >= hi) reinterpret_cast<uint4*>(tile)[i] = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    __syncwarp();
}

// Row `row` of a tile in shared memory <- 32 values at columns [32 c, 32 c + 32), as bf16, in the layout of the copies.
__device__ __forceinline__ void stage_row32(uint8_t* tile, int row, int c, const float (&f)[32]) {
    uint8_t* box = tile + (c >> 1) * kBoxBytes;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<uint4*>(box + swz128(row, (c & 1) * 4 + k)) =
            make_uint4(pack_bf16x2(f[8 * k], f[8 * k + 1]), pack_bf16x2(f[8 * k + 2], f[8 * k + 3]),
                       pack_bf16x2(f[8 * k + 4], f[8 * k + 5]), pack_bf16x2(f[8 * k + 6], f[8 * k + 7]));
}

// ---- geometry -----------------------------------------------------------------------------------------------------

struct Geometry {
    int n_seq, seq_len, heads, kv_heads, group, head_dim, window;  // window: seq_len where there is none
    const int32_t* bounds;
};

// live positions [lo, hi) of generation n
__device__ __forceinline__ void live_range(const Geometry& g, int n, int& lo, int& hi) {
    lo = 0;
    hi = g.seq_len;
    if (g.bounds) {
        lo = min(max(g.bounds[2 * n], 0), g.seq_len);
        hi = min(max(g.bounds[2 * n + 1], lo), g.seq_len);
    }
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

// Tensor map of [n_seq][seq_len][heads][head_dim] bf16 with row pitch `ld` elements, boxes of 128 positions x 64 elements.
bool make_head_map(CUtensorMap* map, const void* base, const rapid_attn_desc_t& d, int heads, int64_t ld);

}  // namespace attn
}  // namespace rapid
