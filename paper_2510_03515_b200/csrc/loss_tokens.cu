// The losses of rapid_losses.h where a row's gradient waits for other rows, or is not wanted: one kernel reads the logits for the
// tokens' log-probabilities, another reads them again and writes the gradient.  Both are one pass at the rate of the memory.
#include <algorithm>

#include "loss_rows.cuh"

namespace rapid {
namespace losses {

namespace {

// ---- log-probabilities -------------------------------------------------------------------------------------------
// A row for each warp (kGroup = 1) or block of four (kGroup = 4), eight 16-byte loads of every thread in flight; some six blocks on
// an SM cover one another's ends.
constexpr int kStatThreads = 128;

// With kKeep the logits stay in L2 as far as they fit, for the gradient's reading.
template <int DT, int kGroup, bool kKeep>
__global__ void __launch_bounds__(kStatThreads, 6)
token_stats_kernel(RowsArgs a, const int32_t* __restrict__ targets, const uint8_t* __restrict__ mask) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int U = 8, kLanes = kGroup * 32;
    __shared__ WarpPart parts[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gt = threadIdx.x % kLanes;
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.w.head = Header{0u, 0u, RAPID_OK, 0};
    const int64_t r = (int64_t)blockIdx.x * (4 / kGroup) + warp / kGroup;
    if (r >= a.n_rows) return;  // the whole block, or warps that meet nobody
    const int y = targets[r];
    const uint8_t state = mask && !mask[r] ? ROW_MASKED : y >= 0 && y < a.vocab ? ROW_OK : ROW_BAD_TOKEN;
    if (gt == 0) {
        a.w.state[r] = state;
        if (state != ROW_OK) a.w.value[r] = 0.0;
    }
    if (state != ROW_OK) return;
    const T* row = static_cast<const T*>(a.logits) + r * a.ld;
    const float z = E::get(row[y]);
    const uint4* rv = reinterpret_cast<const uint4*>(row);
    const int nvec = a.vocab / E::kPer;
    const float off = shift_fraction(kGroup == 1 ? 0 : warp);
    auto load = [](const uint4* at) { return kKeep ? __ldg(at) : ld_stream(at); };
    Part p;
    int v = gt;
    for (; v + (U - 1) * kLanes < nvec; v += U * kLanes) {
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j) q[j] = load(rv + v + j * kLanes);
        p.template vectors<DT, U>(q, off, a.f);
    }
    if (v - lane < nvec) {  // what is left, up to eight vectors of a thread; behind the row: -inf
        constexpr uint32_t kNone = DT == RAPID_BF16 ? 0xff80ff80u : 0xff800000u;
        uint4 q[U];
#pragma unroll
        for (int j = 0; j < U; ++j) q[j] = v + j * kLanes < nvec ? load(rv + v + j * kLanes) : make_uint4(kNone, kNone, kNone, kNone);
        p.template vectors<DT, U>(q, off, a.f);
    }
    const int e = nvec * E::kPer + gt;
    if (e < a.vocab) p.scalar(E::get(row[e]), off, a.f);
    const WarpPart w = warp_part(p, a.f);
    RowStat st;
    if constexpr (kGroup == 1) {
        st = one_part(w, off, part_unit(off), a.f);
    } else {
        if (lane == 0) parts[warp] = w;
        __syncthreads();
        if (warp != 0) return;
        const float off_l = shift_fraction(lane);
        st = join_parts(lane < 4 ? parts[lane] : WarpPart{0.0, -INFINITY, -INFINITY}, off_l, part_unit(off_l), a.f);
    }
    if (lane == 0) {
        a.w.value[r] = ((double)z * a.f.kd - st.lse2) * kLn2D;
        a.w.lse2[r] = st.lse2;
        a.w.row_max[r] = st.max;
    }
}

// ---- gradients ----------------------------------------------------------------------------------------------------
// A warp for each piece of a row, 16 vectors of a lane; it forms the row's constants itself.  Nothing waits for anything.
constexpr int kGradThreads = 256;
constexpr int kPiece = 16 * 32;

template <int DT>
__global__ void __launch_bounds__(kGradThreads)
token_grads_kernel(RowsArgs a, const int32_t* __restrict__ targets, const double* __restrict__ coef, Divisor seq_len, uint32_t pieces, uint32_t total) {
    using E = Elem<DT>;
    using T = typename E::T;
    constexpr int U = 8;
    uint32_t piece = blockIdx.x * (kGradThreads / 32) + (threadIdx.x >> 5);
    if (piece >= total) return;
    piece = total - 1 - piece;  // from the end: what the first reading read last may still be in L2
    const int lane = threadIdx.x & 31;
    const uint32_t r = piece / pieces;
    const int first = (int)(piece - r * pieces) * kPiece;  // first vector
    const int nvec = a.vocab / E::kPer, end = min(first + kPiece, nvec);
    const bool last = first + kPiece >= nvec;
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
    const int64_t row_bytes = (int64_t)a.vocab * (int64_t)elem_size(a.dtype);
    // a warp for a row of up to 16 vectors a lane; longer ones keep four warps' loads in flight
    const bool single = row_bytes <= 8192;
    const unsigned grid = (unsigned)(single ? (a.n_rows + 3) / 4 : a.n_rows);
    auto go = [&](auto kern) {
        kern<<<grid, kStatThreads, 0, stream>>>(a, targets, mask);
        return cudaGetLastError();
    };
    auto by_type = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (keep) return single ? go(token_stats_kernel<DT, 1, true>) : go(token_stats_kernel<DT, 4, true>);
        return single ? go(token_stats_kernel<DT, 1, false>) : go(token_stats_kernel<DT, 4, false>);
    };
    return a.dtype == RAPID_BF16 ? by_type(std::integral_constant<int, RAPID_BF16>{}) : by_type(std::integral_constant<int, RAPID_F32>{});
}

cudaError_t launch_token_grads(const RowsArgs& a, const int32_t* targets, const double* coef, const Divisor& seq_len, cudaStream_t stream) {
    const int64_t nvec = a.vocab / (16 / (int64_t)elem_size(a.dtype));
    const int64_t pieces = std::max<int64_t>(1, (nvec + kPiece - 1) / kPiece), total = pieces * a.n_rows;
    if (total > 0x7fffffffll) return cudaErrorInvalidValue;  // 17 TB of gradient
    const unsigned grid = (unsigned)((total + kGradThreads / 32 - 1) / (kGradThreads / 32));
    auto go = [&](auto kern) {
        kern<<<grid, kGradThreads, 0, stream>>>(a, targets, coef, seq_len, (uint32_t)pieces, (uint32_t)total);
        return cudaGetLastError();
    };
    return a.dtype == RAPID_BF16 ? go(token_grads_kernel<RAPID_BF16>) : go(token_grads_kernel<RAPID_F32>);
}

}  // namespace losses
}  // namespace rapid
