// The losses of rapid_losses.h where a row's gradient waits for other rows, or is not wanted: one kernel reads the logits for the
// tokens' log-probabilities, another reads them again and writes the gradient.  Both are one pass at the rate of the memory.
#include "loss_rows.cuh"

namespace rapid {
namespace losses {

namespace {

// ---- log-probabilities -------------------------------------------------------------------------------------------
// One to four warps for a row; each leaves its part of the row's statistics in memory and is done, without meeting the others.  Whoever
// needs the row joins the parts, a row for each thread.  Eight 16-byte loads of every lane are in flight.
constexpr int kStatThreads = 128;

// With kKeep the logits stay in L2 as far as they fit, for the gradient's reading.
template <int DT, bool kKeep>
__global__ void __launch_bounds__(kStatThreads, 6)
token_stats_kernel(RowsArgs a, const int32_t* __restrict__ targets, const uint8_t* __restrict__ mask, uint32_t pieces, uint32_t total) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int U = 8;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.w.head = Header{0u, 0u, RAPID_OK, 0};
    const uint32_t piece = blockIdx.x * (kStatThreads / 32) + (threadIdx.x >> 5);
    if (piece >= total) return;
    const int lane = threadIdx.x & 31;
    const uint32_t r = pieces == 1 ? piece : piece / pieces, at = piece - r * pieces;
    const int y = targets[r];
    const uint8_t state = mask && !mask[r] ? ROW_MASKED : y >= 0 && y < a.vocab ? ROW_OK : ROW_BAD_TOKEN;
    if (at == 0 && lane == 0) a.w.state[r] = state;
    if (state != ROW_OK) return;
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.ld;
    if (at == 0 && lane == 0) a.w.token_z[r] = E::get(row[y]);
    const uint4* rv = reinterpret_cast<const uint4*>(row);
    const int nvec = a.vocab / E::kPer, lanes = 32 * (int)pieces;  // the row's warps take turns of 32 vectors
    const float off = shift_fraction(at & 31);
    auto load = [](const uint4* p) { return kKeep ? __ldg(p) : ld_stream(p); };
    Part p;
    int v = (int)at * 32 + lane;
    for (; v + (U - 1) * lanes < nvec; v += U * lanes) {
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j) q[j] = load(rv + v + j * lanes);
        p.template vectors<DT, U>(q, off, a.f);
    }
    if (v - lane < nvec) {  // what is left, up to eight vectors of a lane; behind the row: -inf
        constexpr uint32_t kNone = DT == RAPID_BF16 ? 0xff80ff80u : 0xff800000u;
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j) q[j] = v + j * lanes < nvec ? load(rv + v + j * lanes) : make_uint4(kNone, kNone, kNone, kNone);
        p.template vectors<DT, U>(q, off, a.f);
    }
    const int e = nvec * E::kPer + lane;  // fewer columns than a vector has, behind the last one
    if (at == pieces - 1 && e < a.vocab) p.scalar(E::get(row[e]), off, a.f);
    const WarpPart w = warp_part(p, a.f);
    if (lane == 0) a.w.parts[(size_t)r * pieces + at] = w;
}

// ---- gradients ----------------------------------------------------------------------------------------------------
// A warp for each piece of a row, 16 vectors of a lane; it forms the row's constants itself.  Nothing waits for anything.
constexpr int kGradThreads = 256;

template <int DT>
__global__ void __launch_bounds__(kGradThreads, 4)  // (of bf16 three else: 8192 x 32000 280 us instead of 277)
token_grads_kernel(RowsArgs a, const int32_t* __restrict__ targets, const double* __restrict__ coef, Divisor seq_len, uint32_t pieces, uint32_t total) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int U = 8;
    uint32_t piece = blockIdx.x * (kGradThreads / 32) + (threadIdx.x >> 5);
    if (piece >= total) return;
    piece = total - 1 - piece;  // from the end: what the first reading read last may still be in L2
    const int lane = threadIdx.x & 31;
    const uint32_t r = piece / pieces;
    const int first = (int)(piece - r * pieces) * kPieceVecs;  // first vector
    const int nvec = a.vocab / E::kPer, end = min(first + kPieceVecs, nvec);
    const bool last = first + kPieceVecs >= nvec;
    T* out = static_cast<T*>(a.grad) + (int64_t)r * a.ld_grad;
    uint4* ov = reinterpret_cast<uint4*>(out);
    const double g = a.w.state[r] == ROW_OK ? coef[divide(r, seq_len)] : 0.0;
    const int e = nvec * E::kPer + lane;  // columns behind the last whole vector
    if (g == 0.0) {
#pragma unroll 4
        for (int v = first + lane; v < end; v += 32) st_stream(ov + v, make_uint4(0, 0, 0, 0));
        if (last && e < a.vocab) out[e] = E::put(0.f);
        return;
    }
    const T* row = static_cast<const T*>(a.logits) + (int64_t)r * a.ld;
    const uint4* rv = reinterpret_cast<const uint4*>(row);
    const double lse2 = a.w.lse2[r], lp = a.w.value[r];
    const Grad<DT> gr(grad_const<DT>(RowGrad{g, lse2}, a.w.row_max[r], a.f), a.f);
    const int y = targets[r];
    int v = first + lane;
    for (; v - lane + (U - 1) * 32 + 31 < end; v += U * 32) {
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j) q[j] = ld_stream(rv + v + j * 32);
#pragma unroll
        for (int j = 0; j < U; ++j) st_stream(ov + v + j * 32, gr.vector(q[j]));
    }
    {
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (v + j * 32 < end) q[j] = ld_stream(rv + v + j * 32);
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (v + j * 32 < end) st_stream(ov + v + j * 32, gr.vector(q[j]));
    }
    if (last && e < a.vocab) out[e] = gr.one(row[e]);
    __syncwarp();  // then the token's column over its vector
    const int at = y / E::kPer;
    if (lane == 0 && at >= first && (at < end || last)) out[y] = E::put((float)(g * (exp2_short(lp * kLog2eD) - 1.0)));
}

}  // namespace

cudaError_t launch_token_stats(const RowsArgs& a, const int32_t* targets, const uint8_t* mask, bool keep, cudaStream_t stream) {
    const int64_t pieces = stat_pieces(a.vocab, a.dtype), total = pieces * a.n_rows;  // 31 bits: checked
    const unsigned grid = (unsigned)((total + kStatThreads / 32 - 1) / (kStatThreads / 32));
    auto go = [&](auto kern) {
        kern<<<grid, kStatThreads, 0, stream>>>(a, targets, mask, (uint32_t)pieces, (uint32_t)total);
        return cudaGetLastError();
    };
    if (a.dtype == RAPID_BF16) return keep ? go(token_stats_kernel<RAPID_BF16, true>) : go(token_stats_kernel<RAPID_BF16, false>);
    return keep ? go(token_stats_kernel<RAPID_F32, true>) : go(token_stats_kernel<RAPID_F32, false>);
}

cudaError_t launch_token_grads(const RowsArgs& a, const int32_t* targets, const double* coef, const Divisor& seq_len, cudaStream_t stream) {
    const int64_t pieces = grad_pieces(a.vocab, a.dtype), total = pieces * a.n_rows;  // 31 bits: checked
    const unsigned grid = (unsigned)((total + kGradThreads / 32 - 1) / (kGradThreads / 32));
    auto go = [&](auto kern) {
        kern<<<grid, kGradThreads, 0, stream>>>(a, targets, coef, seq_len, (uint32_t)pieces, (uint32_t)total);
        return cudaGetLastError();
    };
    return a.dtype == RAPID_BF16 ? go(token_grads_kernel<RAPID_BF16>) : go(token_grads_kernel<RAPID_F32>);
}

}  // namespace losses
}  // namespace rapid
