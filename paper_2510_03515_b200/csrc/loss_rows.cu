// The rows of the losses of rapid_losses.h: one block for each row, which reads it twice and writes its gradient.
#include "loss_rows.cuh"

namespace rapid {
namespace losses {

namespace {

constexpr int kThreads = 256;

template <int DT, class Op>
__global__ void __launch_bounds__(kThreads) rows_kernel(RowsArgs a, Op op) {
    using E = Elem<DT>;
    using T = typename E::T;
    extern __shared__ uint32_t left_out[];  // a bit for each column that the sum leaves out
    __shared__ WarpPart parts[kThreads / 32];
    __shared__ float z[kMaxList], value[kMaxList];
    __shared__ RowGrad grad;
    __shared__ float row_max;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool ex = exclude(op) && !a.known;
    const int nvec = a.vocab / E::kPer;
    long long rows = 0;
    if (warp == 0 && op_counts(op)) rows = rows_that_count(op_counts(op), op_blocks(op));
    if (ex)
        for (int i = tid; i < (a.vocab + 31) / 32; i += kThreads) left_out[i] = 0;
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        const T* row = static_cast<const T*>(a.logits) + r * a.ld;
        T* out = static_cast<T*>(a.grad) + r * a.ld_grad;
        if (a.w.state[r] != ROW_OK) {
            if (a.grad)
                for (int v = tid; v < a.vocab; v += kThreads) out[v] = E::put(0.f);
            if (!a.known && tid == 0) a.w.value[r] = 0.0;
            continue;
        }
        const int n_list = list_size(op);
        __syncthreads();
        for (int j = tid; j < n_list; j += kThreads) {
            const int v = column(op, r, j);
            if (v >= 0) {
                z[j] = E::get(row[v]);
                if (ex) atomicOr(&left_out[v >> 5], 1u << (v & 31));
            }
        }
        __syncthreads();
        RowStat st;
        if (!a.known) {
            const float off = shift_fraction(warp);
            Part p;
            for (int v = tid; v < nvec; v += kThreads) {
                uint4 q[1] = {reinterpret_cast<const uint4*>(row)[v]};
                if (ex) {
                    T* e = reinterpret_cast<T*>(q);
                    const uint32_t bits = left_out[v * E::kPer >> 5] >> (v * E::kPer & 31);
#pragma unroll
                    for (int i = 0; i < E::kPer; ++i)
                        if (bits >> i & 1u) e[i] = E::put(-INFINITY);
                }
                p.template vectors<DT, 1>(q, off, a.f);
            }
            const int e = nvec * E::kPer + tid;
            if (e < a.vocab && !(ex && (left_out[e >> 5] >> (e & 31) & 1u))) p.scalar(E::get(row[e]), off, a.f);
            const WarpPart w = warp_part(p, a.f);
            if (lane == 0) parts[warp] = w;
            __syncthreads();
            if (warp == 0) {
                WarpPart mine{-INFINITY, -INFINITY, 0.0};
                if (lane < kThreads / 32) mine = parts[lane];
                st = join_parts(mine, a.f);
            }
        } else {
            st.lse2 = a.w.lse2[r];
            st.max = a.w.row_max[r];
        }
        if (warp == 0) {
            const RowGrad g = finish(op, a, r, st, z, value, rows);
            if (lane == 0) {
                grad = g;
                row_max = st.max;
            }
        }
        __syncthreads();
        if (ex)
            for (int j = tid; j < n_list; j += kThreads) {
                const int v = column(op, r, j);
                if (v >= 0) left_out[v >> 5] = 0;
            }
        if (a.grad) {
            Grad<DT> gr;
            gr.set(grad.a, grad.lse2, row_max, a.f);
            for (int v = tid; v < nvec; v += kThreads)
                reinterpret_cast<uint4*>(out)[v] = gr.vector(reinterpret_cast<const uint4*>(row)[v]);
            const int e = nvec * E::kPer + tid;
            if (e < a.vocab) out[e] = gr.one(row[e]);
            __syncthreads();
            for (int j = tid; j < n_list; j += kThreads) {
                const int v = column(op, r, j);
                if (v >= 0) out[v] = E::put(value[j]);
            }
        }
    }
}

template <class Op>
cudaError_t launch(const RowsArgs& a, const Op& op, bool ex, int sm_count, cudaStream_t stream) {
    const size_t smem = ex ? (size_t)(a.vocab + 31) / 32 * 4 : 0;
    const int64_t grid = a.n_rows < 8ll * sm_count ? a.n_rows : 8ll * sm_count;
    auto go = [&](auto kern) -> cudaError_t {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        kern<<<(unsigned)grid, kThreads, smem, stream>>>(a, op);
        return cudaGetLastError();
    };
    return a.dtype == RAPID_BF16 ? go(rows_kernel<RAPID_BF16, Op>) : go(rows_kernel<RAPID_F32, Op>);
}

}  // namespace

cudaError_t launch_rows(const RowsArgs& a, const ClipOp& op, int sm_count, cudaStream_t stream) { return launch(a, op, false, sm_count, stream); }
cudaError_t launch_rows(const RowsArgs& a, const PrefOp& op, int sm_count, cudaStream_t stream) { return launch(a, op, false, sm_count, stream); }
cudaError_t launch_rows(const RowsArgs& a, const DistillOp& op, int sm_count, cudaStream_t stream) {
    return launch(a, op, op.tail != 0 && !a.known, sm_count, stream);
}

}  // namespace losses
}  // namespace rapid
