// Norms of query and key heads with the rotation by position, and the gradient.  One pass over the data, bound by HBM
// bytes.
//
// A lane holds 16 elements of a head as two vectors of 8 whose elements form rotation pairs with one another (halves: 8 at
// i and 8 at i + rot_dim / 2; interleaved: 16 neighbours), so a rotation needs no exchange between lanes; the lanes of
// a head (head_dim / 16 rounded up to a power of two) exchange only the sums of the norm.  A group of lanes stays on one
// row and walks its heads, so the 8 angles of a lane are formed once for all heads.  Angles are products in double,
// reduced to a fraction of a turn in double (a float angle at position 100 000 is off by 4e-3), then sine and cosine in
// float.
#include <math.h>

#include "policy_ops.cuh"

namespace rapid {
namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHeadDim = 256;

struct QkArgs {
    int64_t n_rows;
    int seq_len, heads_q, heads, head_dim, rot_dim;  // heads = queries and keys together
    int lanes_log2;                                  // lanes of a head
    int parts, per_part;                             // a row's heads are split over `parts` groups
    uint32_t flags;
    float eps;
    int64_t ld_q, ld_k, ld_q_out, ld_k_out, ld_dq, ld_dk;
    const float *q_weight, *k_weight, *inv_freq;
    const int32_t* positions;
    const uint8_t* mask;
};

// Where a lane's two vectors of 8 elements lie in a head, and whether they rotate.
struct Place {
    int a, b, angle;  // offsets of the vectors, first angle; angle < 0: no rotation
    bool on;
};

__device__ __forceinline__ Place place_of(const QkArgs& p, int u) {
    Place x;
    x.on = u < p.head_dim / 16;
    const int turning = p.rot_dim / 16;
    if (u < turning && !(p.flags & RAPID_QK_INTERLEAVED)) {
        x.a = 8 * u;
        x.b = p.rot_dim / 2 + 8 * u;
    } else {
        x.a = 16 * u;
        x.b = 16 * u + 8;
    }
    x.angle = u < turning ? 8 * u : -1;
    return x;
}

__device__ __forceinline__ void angles(const QkArgs& p, const Place& x, int64_t r, float (&cs)[8], float (&sn)[8]) {
    if (x.angle < 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = 1.f, sn[j] = 0.f;
        return;
    }
    const double pos = (double)(p.positions ? p.positions[r] : (int32_t)(r % p.seq_len));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        double t = pos * (double)p.inv_freq[x.angle + j] * 0.15915494309189533577;  // turns: angle / (2 pi)
        t -= rint(t);
        sincospif((float)(2.0 * t), &sn[j], &cs[j]);
    }
}

// (a_i, b_i) -> (a_i c - b_i s, a_i s + b_i c) over the lane's 8 pairs; halves: a and b, interleaved: neighbours
__device__ __forceinline__ void rotate(bool interleaved, float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a0 = a[2 * j], a1 = a[2 * j + 1], b0 = b[2 * j], b1 = b[2 * j + 1];
            a[2 * j] = a0 * cs[j] - a1 * sn[j];
            a[2 * j + 1] = a0 * sn[j] + a1 * cs[j];
            b[2 * j] = b0 * cs[4 + j] - b1 * sn[4 + j];
            b[2 * j + 1] = b0 * sn[4 + j] + b1 * cs[4 + j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float x = a[j], y = b[j];
            a[j] = x * cs[j] - y * sn[j];
            b[j] = x * sn[j] + y * cs[j];
        }
    }
}

__device__ __forceinline__ float group_sum(float v, int lanes_log2) {
    for (int o = 1; o < (1 << lanes_log2); o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The factors of the two norms, in shared memory: [0] queries, [1] keys.
__device__ __forceinline__ void load_weights(const QkArgs& p, float (*w)[kMaxHeadDim]) {
    const float add = (p.flags & RAPID_QK_UNIT_OFFSET) ? 1.f : 0.f;
    if (!(p.flags & RAPID_QK_NO_NORM))
        for (int i = threadIdx.x; i < p.head_dim; i += kThreads) {
            w[0][i] = p.q_weight[i] + add;
            w[1][i] = p.k_weight[i] + add;
        }
    __syncthreads();
}

constexpr int kHeadsAhead = 4;  // heads whose loads are in flight together

template <class T>
__global__ void __launch_bounds__(kThreads)
qk_fwd_kernel(QkArgs p, const T* q, const T* k, T* q_out, T* k_out) {
    __shared__ float w[2][kMaxHeadDim];
    load_weights(p, w);
    const int lane = threadIdx.x & 31;
    const int64_t group = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> p.lanes_log2;
    const bool norm = !(p.flags & RAPID_QK_NO_NORM), inter = (p.flags & RAPID_QK_INTERLEAVED) != 0;
    const int64_t r = group / p.parts;
    const int h0 = (int)(group - r * p.parts) * p.per_part;
    const bool row = r < p.n_rows;
    const int h1 = row ? min(h0 + p.per_part, p.heads) : h0;
    const bool live = row && (p.mask == nullptr || p.mask[r] != 0);
    const Place x = place_of(p, lane & ((1 << p.lanes_log2) - 1));
    float cs[8], sn[8];
    if (live && x.on) angles(p, x, r, cs, sn);
    // the same number of turns in every lane of the warp: the sums exchange over whole warps
    for (int hh = 0; hh < p.per_part; hh += kHeadsAhead) {
        Vec8<T> va[kHeadsAhead], vb[kHeadsAhead];
#pragma unroll
        for (int u = 0; u < kHeadsAhead; ++u) {
            const int h = h0 + hh + u;
            if (hh + u < p.per_part && h < h1 && live && x.on) {
                const T* src = h < p.heads_q ? q + r * p.ld_q + h * p.head_dim : k + r * p.ld_k + (h - p.heads_q) * p.head_dim;
                va[u].load(src + x.a);
                vb[u].load(src + x.b);
            }
        }
#pragma unroll
        for (int u = 0; u < kHeadsAhead; ++u) {
            const int h = h0 + hh + u;
            const bool have = hh + u < p.per_part && h < h1 && x.on;
            float a[8], b[8];
            if (have && live) {
                va[u].get(a);
                vb[u].get(b);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.f;
            }
            if (norm) {
                float sq = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sq += a[j] * a[j] + b[j] * b[j];
                sq = group_sum(sq, p.lanes_log2);
                const float rstd = 1.f / sqrtf(sq / (float)p.head_dim + p.eps);
                const float* wt = w[h < p.heads_q ? 0 : 1];
                if (have && live) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        a[j] *= rstd * wt[x.a + j];
                        b[j] *= rstd * wt[x.b + j];
                    }
                }
            }
            if (have) {
                if (live && x.angle >= 0) rotate(inter, a, b, cs, sn);
                T* dst = h < p.heads_q ? q_out + r * p.ld_q_out + h * p.head_dim
                                       : k_out + r * p.ld_k_out + (h - p.heads_q) * p.head_dim;
                Vec8<T>::store(dst + x.a, a);
                Vec8<T>::store(dst + x.b, b);
            }
        }
    }
}

// The gradient.  A group takes rows group, group + groups, ... and keeps its lanes' share of the two weight gradients in
// registers; a block adds its groups in order and leaves one partial sum, which qk_weight_grad_kernel adds in order.
template <class T>
__global__ void __launch_bounds__(kThreads)
qk_bwd_kernel(QkArgs p, const T* q, const T* k, const T* dq_out, const T* dk_out, T* dq, T* dk, float* __restrict__ partial) {
    __shared__ float w[2][kMaxHeadDim];
    __shared__ float part[kThreads][17];
    load_weights(p, w);
    const int lane = threadIdx.x & 31;
    const int lanes = 1 << p.lanes_log2;
    const int64_t groups = (int64_t)gridDim.x * (kThreads >> p.lanes_log2);
    const int64_t group = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> p.lanes_log2;
    const bool norm = !(p.flags & RAPID_QK_NO_NORM), inter = (p.flags & RAPID_QK_INTERLEAVED) != 0;
    const Place x = place_of(p, lane & (lanes - 1));
    float dw[2][16] = {};
    const int64_t units = p.n_rows * p.parts;
    const int64_t turns = (units + groups - 1) / groups;
    for (int64_t turn = 0; turn < turns; ++turn) {
        const int64_t unit = group + turn * groups;
        const int64_t r = unit / p.parts;
        const int h0 = (int)(unit - r * p.parts) * p.per_part;
        const bool row = unit < units;
        const int h1 = row ? min(h0 + p.per_part, p.heads) : h0;
        const bool live = row && (p.mask == nullptr || p.mask[r] != 0);
        float cs[8], sn[8];
        if (live && x.on) {
            angles(p, x, r, cs, sn);
#pragma unroll
            for (int j = 0; j < 8; ++j) sn[j] = -sn[j];  // rotate back
        }
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {  // queries, keys: the sums of the weight gradients stay in registers
            const int from = kind == 0 ? 0 : p.heads_q, to = kind == 0 ? p.heads_q : p.heads;
#pragma unroll 1
            for (int hh = 0; hh < p.per_part; hh += 2) {
                // whole warps skip turns that hold no head of this kind
                const bool any = h0 + hh < min(h1, to) && h0 + hh + 1 >= from;
                if (!__any_sync(0xffffffffu, any)) continue;
                Vec8<T> xa[2], xb[2], ya[2], yb[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int h = h0 + hh + u;
                    if (hh + u < p.per_part && h >= from && h < min(h1, to) && live && x.on) {
                        const T* src = kind == 0 ? q + r * p.ld_q + h * p.head_dim : k + r * p.ld_k + (h - from) * p.head_dim;
                        const T* g = kind == 0 ? dq_out + r * p.ld_q_out + h * p.head_dim
                                               : dk_out + r * p.ld_k_out + (h - from) * p.head_dim;
                        if (norm) {
                            xa[u].load(src + x.a);
                            xb[u].load(src + x.b);
                        }
                        ya[u].load(g + x.a);
                        yb[u].load(g + x.b);
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int h = h0 + hh + u;
                    const bool have = hh + u < p.per_part && h >= from && h < min(h1, to) && x.on;
                    const bool on = have && live;
                    float a[8], b[8], ga[8], gb[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) a[j] = b[j] = ga[j] = gb[j] = 0.f;
                    if (on) {
                        ya[u].get(ga);
                        yb[u].get(gb);
                        if (x.angle >= 0) rotate(inter, ga, gb, cs, sn);
                    }
                    if (norm) {
                        if (on) {
                            xa[u].get(a);
                            xb[u].get(b);
                        }
                        float sq = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) sq += a[j] * a[j] + b[j] * b[j];
                        sq = group_sum(sq, p.lanes_log2);
                        const float rstd = 1.f / sqrtf(sq / (float)p.head_dim + p.eps);
                        float dot = 0.f;
                        if (on) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                a[j] *= rstd;
                                b[j] *= rstd;
                                dw[kind][j] += ga[j] * a[j];
                                dw[kind][8 + j] += gb[j] * b[j];
                                ga[j] *= w[kind][x.a + j];
                                gb[j] *= w[kind][x.b + j];
                                dot += ga[j] * a[j] + gb[j] * b[j];
                            }
                        }
                        dot = group_sum(dot, p.lanes_log2) / (float)p.head_dim;
                        if (on) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                ga[j] = (ga[j] - a[j] * dot) * rstd;
                                gb[j] = (gb[j] - b[j] * dot) * rstd;
                            }
                        }
                    }
                    if (have) {
                        T* dst = kind == 0 ? dq + r * p.ld_dq + h * p.head_dim : dk + r * p.ld_dk + (h - from) * p.head_dim;
                        Vec8<T>::store(dst + x.a, ga);
                        Vec8<T>::store(dst + x.b, gb);
                    }
                }
            }
        }
    }
    if (!norm) return;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 16; ++j) part[threadIdx.x][j] = dw[kind][j];
        __syncthreads();
        // thread (lane u of a group, element j): the sum over the block's groups
        for (int i = threadIdx.x; i < lanes * 16; i += kThreads) {
            const int u = i >> 4, j = i & 15;
            const Place y = place_of(p, u);
            if (!y.on) continue;
            float sum = 0.f;
            for (int g = 0; g < (kThreads >> p.lanes_log2); ++g) sum += part[g * lanes + u][j];
            partial[((size_t)blockIdx.x * 2 + kind) * kMaxHeadDim + (j < 8 ? y.a + j : y.b + j - 8)] = sum;
        }
    }
}

// One block for each kind and 8 columns: 32 threads a column each add every 32nd partial sum, then the 32 sums in order.
__global__ void __launch_bounds__(256)
qk_weight_grad_kernel(int blocks, int head_dim, const float* __restrict__ partial, float* __restrict__ dq_weight,
                      float* __restrict__ dk_weight) {
    __shared__ double part[8][33];
    const int kind = blockIdx.y, col = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int c = blockIdx.x * 8 + col;
    double sum = 0.0;
    for (int b = slice; b < blocks; b += 32) sum += (double)partial[((size_t)b * 2 + kind) * kMaxHeadDim + c];
    part[col][slice] = sum;
    __syncthreads();
    if (threadIdx.x < 8) {
        double total = 0.0;
        for (int i = 0; i < 32; ++i) total += part[threadIdx.x][i];
        (kind == 0 ? dq_weight : dk_weight)[blockIdx.x * 8 + threadIdx.x] = (float)total;
    }
}

// ---- host side ------------------------------------------------------------------------------------------------

constexpr int kMaxBwdBlocks = 1024;

rapid_status_t check_qk(const rapid_qk_desc_t* d, bool bwd) {
    if (!d || d->n_seq <= 0 || d->seq_len <= 0 || d->n_q_heads <= 0 || d->n_k_heads <= 0 || d->reserved != 0)
        return RAPID_ERR_INVALID_ARG;
    if (d->dtype != RAPID_F32 && d->dtype != RAPID_BF16) return RAPID_ERR_INVALID_ARG;
    if (d->flags & ~(uint32_t)(RAPID_QK_NO_NORM | RAPID_QK_UNIT_OFFSET | RAPID_QK_INTERLEAVED)) return RAPID_ERR_INVALID_ARG;
    if (d->head_dim <= 0 || d->rot_dim <= 0 || d->rot_dim > d->head_dim) return RAPID_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || !isfinite(d->eps)) return RAPID_ERR_INVALID_ARG;
    if (d->head_dim % 16 != 0 || d->head_dim > kMaxHeadDim || d->rot_dim % 16 != 0) return RAPID_ERR_UNSUPPORTED;
    if (d->n_q_heads > 4096 || d->n_k_heads > 4096) return RAPID_ERR_UNSUPPORTED;
    if ((int64_t)d->n_seq * d->seq_len > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;
    const int64_t wq = (int64_t)d->n_q_heads * d->head_dim, wk = (int64_t)d->n_k_heads * d->head_dim;
    if (d->ld_q < wq || d->ld_q_out < wq || d->ld_k < wk || d->ld_k_out < wk) return RAPID_ERR_INVALID_ARG;
    const int64_t most = 1ll << 31;
    if (d->ld_q > most || d->ld_k > most || d->ld_q_out > most || d->ld_k_out > most) return RAPID_ERR_UNSUPPORTED;
    const int64_t unit = 16 / (int64_t)elem_size(d->dtype);
    if (d->ld_q % unit || d->ld_k % unit || d->ld_q_out % unit || d->ld_k_out % unit) return RAPID_ERR_ALIGNMENT;
    if (bwd) {
        if (d->ld_dq < wq || d->ld_dk < wk) return RAPID_ERR_INVALID_ARG;
        if (d->ld_dq > most || d->ld_dk > most) return RAPID_ERR_UNSUPPORTED;
        if (d->ld_dq % unit || d->ld_dk % unit) return RAPID_ERR_ALIGNMENT;
    }
    return RAPID_OK;
}

QkArgs make_args(const rapid_qk_desc_t& d, const float* q_weight, const float* k_weight, const float* inv_freq,
                 const int32_t* positions, const uint8_t* mask, int sms) {
    QkArgs p{};
    p.n_rows = (int64_t)d.n_seq * d.seq_len;
    p.seq_len = d.seq_len;
    p.heads_q = d.n_q_heads;
    p.heads = d.n_q_heads + d.n_k_heads;
    p.head_dim = d.head_dim;
    p.rot_dim = d.rot_dim;
    while ((16 << p.lanes_log2) < d.head_dim) ++p.lanes_log2;
    // Few rows: split a row's heads over groups until there are about 16 warps for each SM.
    const int64_t groups = (int64_t)sms * 16 * (32 >> p.lanes_log2);
    int64_t parts = (groups + p.n_rows - 1) / p.n_rows;
    if (parts > p.heads) parts = p.heads;
    p.per_part = (int)((p.heads + parts - 1) / parts);
    p.parts = (p.heads + p.per_part - 1) / p.per_part;
    p.flags = d.flags;
    p.eps = d.eps;
    p.ld_q = d.ld_q;
    p.ld_k = d.ld_k;
    p.ld_q_out = d.ld_q_out;
    p.ld_k_out = d.ld_k_out;
    p.ld_dq = d.ld_dq;
    p.ld_dk = d.ld_dk;
    p.q_weight = q_weight;
    p.k_weight = k_weight;
    p.inv_freq = inv_freq;
    p.positions = positions;
    p.mask = mask;
    return p;
}

int64_t blocks_for(const QkArgs& p) {
    const int64_t per_block = kThreads >> p.lanes_log2;
    return (p.n_rows * p.parts + per_block - 1) / per_block;
}

template <class T>
void run_bwd(const QkArgs& p, int grid, const void* q, const void* k, const void* dq_out, const void* dk_out, void* dq, void* dk,
             float* partial, cudaStream_t st) {
    qk_bwd_kernel<T><<<grid, kThreads, 0, st>>>(p, static_cast<const T*>(q), static_cast<const T*>(k),
                                                static_cast<const T*>(dq_out), static_cast<const T*>(dk_out),
                                                static_cast<T*>(dq), static_cast<T*>(dk), partial);
}

}  // namespace
}  // namespace policy
}  // namespace rapid

using namespace rapid;
using namespace rapid::policy;

extern "C" rapid_status_t rapid_qk_norm_rope_fwd(const rapid_qk_desc_t* desc, const void* q, const void* k,
                                                 const float* q_weight, const float* k_weight, const float* inv_freq,
                                                 const int32_t* positions, const uint8_t* mask, void* q_out, void* k_out,
                                                 void* stream) {
    rapid_status_t s = check_qk(desc, false);
    if (s != RAPID_OK) return s;
    const rapid_qk_desc_t& d = *desc;
    if (!q || !k || !inv_freq || !q_out || !k_out) return RAPID_ERR_INVALID_ARG;
    if (!(d.flags & RAPID_QK_NO_NORM) && (!q_weight || !k_weight)) return RAPID_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16)) return RAPID_ERR_ALIGNMENT;
    const int64_t n = (int64_t)d.n_seq * d.seq_len, wq = (int64_t)d.n_q_heads * d.head_dim, wk = (int64_t)d.n_k_heads * d.head_dim;
    const size_t es = elem_size(d.dtype);
    const bool q_in_place = q == q_out && d.ld_q == d.ld_q_out, k_in_place = k == k_out && d.ld_k == d.ld_k_out;
    if (rows_overlap(q_out, wq, d.ld_q_out, k_out, wk, d.ld_k_out, n, es) ||
        (!q_in_place && rows_overlap(q, wq, d.ld_q, q_out, wq, d.ld_q_out, n, es)) ||
        (!k_in_place && rows_overlap(k, wk, d.ld_k, k_out, wk, d.ld_k_out, n, es)) ||
        rows_overlap(q, wq, d.ld_q, k_out, wk, d.ld_k_out, n, es) || rows_overlap(k, wk, d.ld_k, q_out, wq, d.ld_q_out, n, es))
        return RAPID_ERR_INVALID_ARG;
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    const QkArgs p = make_args(d, q_weight, k_weight, inv_freq, positions, mask, sms);
    const int64_t grid = blocks_for(p);
    if (grid > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d.dtype == RAPID_BF16)
        qk_fwd_kernel<uint16_t><<<(unsigned)grid, kThreads, 0, st>>>(p, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k),
                                                                    static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_out));
    else
        qk_fwd_kernel<float><<<(unsigned)grid, kThreads, 0, st>>>(p, static_cast<const float*>(q), static_cast<const float*>(k),
                                                                 static_cast<float*>(q_out), static_cast<float*>(k_out));
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}

extern "C" rapid_status_t rapid_qk_norm_rope_bwd_workspace_bytes(const rapid_qk_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    rapid_status_t s = check_qk(desc, true);
    if (s != RAPID_OK) return s;
    *bytes = (size_t)kMaxBwdBlocks * 2 * kMaxHeadDim * sizeof(float);
    return RAPID_OK;
}

extern "C" rapid_status_t rapid_qk_norm_rope_bwd(const rapid_qk_desc_t* desc, const void* q, const void* k, const float* q_weight,
                                                 const float* k_weight, const float* inv_freq, const int32_t* positions,
                                                 const uint8_t* mask, const void* dq_out, const void* dk_out, void* dq, void* dk,
                                                 float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes,
                                                 void* stream) {
    rapid_status_t s = check_qk(desc, true);
    if (s != RAPID_OK) return s;
    const rapid_qk_desc_t& d = *desc;
    const bool norm = !(d.flags & RAPID_QK_NO_NORM);
    if (!q || !k || !inv_freq || !dq_out || !dk_out || !dq || !dk) return RAPID_ERR_INVALID_ARG;
    if (norm && (!q_weight || !k_weight || !dq_weight || !dk_weight)) return RAPID_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(dq_out, 16) || !aligned(dk_out, 16) || !aligned(dq, 16) || !aligned(dk, 16))
        return RAPID_ERR_ALIGNMENT;
    const int64_t n = (int64_t)d.n_seq * d.seq_len, wq = (int64_t)d.n_q_heads * d.head_dim, wk = (int64_t)d.n_k_heads * d.head_dim;
    const size_t es = elem_size(d.dtype);
    const bool q_in_place = dq == dq_out && d.ld_dq == d.ld_q_out, k_in_place = dk == dk_out && d.ld_dk == d.ld_k_out;
    // dq and dk against each other and against every input but the gradient that each may replace
    if (rows_overlap(dq, wq, d.ld_dq, dk, wk, d.ld_dk, n, es) || rows_overlap(dq, wq, d.ld_dq, q, wq, d.ld_q, n, es) ||
        rows_overlap(dq, wq, d.ld_dq, k, wk, d.ld_k, n, es) || rows_overlap(dk, wk, d.ld_dk, q, wq, d.ld_q, n, es) ||
        rows_overlap(dk, wk, d.ld_dk, k, wk, d.ld_k, n, es) || rows_overlap(dq, wq, d.ld_dq, dk_out, wk, d.ld_k_out, n, es) ||
        rows_overlap(dk, wk, d.ld_dk, dq_out, wq, d.ld_q_out, n, es) ||
        (!q_in_place && rows_overlap(dq, wq, d.ld_dq, dq_out, wq, d.ld_q_out, n, es)) ||
        (!k_in_place && rows_overlap(dk, wk, d.ld_dk, dk_out, wk, d.ld_k_out, n, es)))
        return RAPID_ERR_INVALID_ARG;
    size_t need = 0;
    if ((s = rapid_qk_norm_rope_bwd_workspace_bytes(desc, &need)) != RAPID_OK) return s;
    if (norm && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return RAPID_ERR_WORKSPACE;
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    const QkArgs p = make_args(d, q_weight, k_weight, inv_freq, positions, mask, sms);
    int64_t grid = blocks_for(p);
    int64_t most = (int64_t)sms * 2 * 2;  // two resident blocks an SM, twice over
    if (most > kMaxBwdBlocks) most = kMaxBwdBlocks;
    if (grid > most) grid = most;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float* partial = static_cast<float*>(workspace);
    if (d.dtype == RAPID_BF16) run_bwd<uint16_t>(p, (int)grid, q, k, dq_out, dk_out, dq, dk, partial, st);
    else run_bwd<float>(p, (int)grid, q, k, dq_out, dk_out, dq, dk, partial, st);
    if (norm)
        qk_weight_grad_kernel<<<dim3((unsigned)(d.head_dim / 8), 2), 256, 0, st>>>((int)grid, d.head_dim, partial, dq_weight, dk_weight);
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
