// Norms of query and key heads with the rotation by position, and the gradient.  One pass over the data, bound by HBM
// bytes.
//
// A lane holds 16 elements of a head as two vectors of 8 whose elements form rotation pairs with one another (halves: 8 at
// i and 8 at i + rot_dim / 2; interleaved: 16 neighbours), so a rotation needs no exchange between lanes; the lanes of
// a head (head_dim / 16 rounded up to a power of two: a group) exchange only the sums of the norm.  A group stays on one row
// and takes every few of its heads, several of them in flight; the angles of a warp's rows are formed once for all heads, in
// shared memory, by the warp itself while its first loads are under way, so no warp waits for another.
// Angles are products in double, reduced to a fraction of a turn in double (a float angle at position 100 000 is off by
// 4e-3), then sine and cosine in float.
//
// What has to be saved here is instructions: rows and pointers are worked out once for each group, the arithmetic is on packed
// pairs of floats, and lanes without a head run along instead of branching.  64 x 1024 rows of 12 + 2 heads of 128, bf16, over
// a third of them masked: forward 145 us with a division for each head and one float operation at a time, 114 packed, 99 with
// the grid walking its tiles, 95 without block barriers, 82 with eight heads in flight and no branches (4.7 TB/s); the
// gradient 273, 154, 149 and, with queries and keys in blocks of their own, half the weight sums a lane and all groups
// busy on the keys' few heads, 120 (4.4 TB/s).  Three blocks an SM spill registers: 112 and 200 us.  Now 45 % of the issue slots are
// used, and what the 15 warps of an SM have in flight bounds both.  Float, 16 x 1024: 42 and 68 us; rotation alone, bf16, 64 x 1024: 72
// and 82.
#include <math.h>

#include "policy_ops.cuh"

namespace rapid {
namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHeadDim = 256;

template <class T>
constexpr int kAhead = sizeof(T) == 2 ? 8 : 4;  // forward: heads of a group in flight, at most

struct QkArgs {
    int64_t n_rows;
    int seq_len, heads_q, heads, head_dim, rot_dim;  // heads = queries and keys together
    int lanes_log2;  // lanes of a head (a template argument of the kernels): 2, 3 or 4
    int per_row;     // groups on one row (forward)
    uint32_t flags;
    float eps, inv_dim;
    int64_t ld_q, ld_k, ld_q_out, ld_k_out;
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

constexpr int kWarpAngles = 32 * 8;

// What a block keeps in shared memory.
struct Shared {
    float weight[2][kMaxHeadDim];  // factors of the norm: queries, keys
    double turns[kMaxHeadDim / 2]; // inv_freq / (2 pi)
    // [warp][row of the warp][rot_dim / 2]; a group of lanes has at most 8 angles a lane
    float cs[kThreads / 32][kWarpAngles], sn[kThreads / 32][kWarpAngles];
};

__device__ __forceinline__ bool row_live(const QkArgs& p, int64_t r) { return r < p.n_rows && (p.mask == nullptr || p.mask[r] != 0); }

// The rows that a warp's groups work on are [first, first + count), counted from the tile's first.
struct WarpRows {
    int first, count;
};
template <int LANES_LOG2>
__device__ __forceinline__ WarpRows warp_rows(int per_row) {
    const int group0 = (threadIdx.x & ~31) >> LANES_LOG2, last = (threadIdx.x | 31) >> LANES_LOG2;
    WarpRows w;
    w.first = group0 / per_row;
    w.count = last / per_row - w.first + 1;
    return w;
}

// Position of row r for the lane that asks for it.
__device__ __forceinline__ double position(const QkArgs& p, int64_t r) {
    if (r >= p.n_rows) return 0.0;
    return (double)(p.positions ? p.positions[r] : (int32_t)((uint32_t)r % (uint32_t)p.seq_len));
}

// Sines and cosines of a warp's rows; lane i < count has the position of row i.
__device__ __forceinline__ void angles(const QkArgs& p, Shared& sm, int count, double pos) {
    const int n = p.rot_dim / 2, lane = threadIdx.x & 31;  // 8 <= n <= 128
    float *cs = sm.cs[threadIdx.x >> 5], *sn = sm.sn[threadIdx.x >> 5];
    int row = 0, k = lane;
    for (int i = 0; i < count * n; i += 32) {
        while (k >= n) {
            k -= n;
            ++row;
        }
        const double at = __shfl_sync(0xffffffffu, pos, row & 31);
        if (row < count) {
            double t = at * sm.turns[k];
            t -= rint(t);
            sincospif((float)(2.0 * t), &sn[i + lane], &cs[i + lane]);
        }
        k += 32;
    }
}

// Eight floats as four packed pairs.
struct Pairs {
    uint64_t v[4];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = 0;
    }
    __device__ __forceinline__ void from(const float* src) {  // shared memory, 16-byte aligned
        const ulonglong2 x = reinterpret_cast<const ulonglong2*>(src)[0], y = reinterpret_cast<const ulonglong2*>(src)[1];
        v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
    }
    template <class T>
    __device__ __forceinline__ void from(const Vec8<T>& x) {
        float f[8];
        x.get(f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f32x2(f[2 * j], f[2 * j + 1]);
    }
    template <class T>
    __device__ __forceinline__ void store(T* p) const {
        float f[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) f32x2_split(v[j], f[2 * j], f[2 * j + 1]);
        Vec8<T>::store(p, f);
    }
    __device__ __forceinline__ void times(const Pairs& o) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f32x2_mul(v[j], o.v[j]);
    }
    __device__ __forceinline__ void times(float x) {
        const uint64_t y = f32x2(x, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f32x2_mul(v[j], y);
    }
};
__device__ __forceinline__ uint64_t negated(uint64_t x) { return x ^ 0x8000000080000000ull; }

// The angles of a lane's 8 pairs; turning back is turning by the negative angle.
template <bool INTER>
struct Angles {
    Pairs cs, sn;
    __device__ __forceinline__ void from(const float* c, const float* s, bool back) {
        cs.from(c);
        sn.from(s);
        if (back) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sn.v[j] = negated(sn.v[j]);
        }
    }
};

// (a_i, b_i) -> (a_i c - b_i s, a_i s + b_i c) over the lane's 8 pairs; halves: a and b, interleaved: neighbours
template <bool INTER>
__device__ __forceinline__ void rotate(Pairs& a, Pairs& b, const Angles<INTER>& t) {
    if constexpr (INTER) {
        auto turn = [](Pairs& x, uint64_t c0, uint64_t s0, uint64_t c1, uint64_t s1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float u, v, ca, cb, sa, sb;
                f32x2_split(x.v[j], u, v);
                f32x2_split(j < 2 ? c0 : c1, ca, cb);
                f32x2_split(j < 2 ? s0 : s1, sa, sb);
                const float c = j & 1 ? cb : ca, s = j & 1 ? sb : sa;
                x.v[j] = f32x2(u * c - v * s, u * s + v * c);
            }
        };
        turn(a, t.cs.v[0], t.sn.v[0], t.cs.v[1], t.sn.v[1]);
        turn(b, t.cs.v[2], t.sn.v[2], t.cs.v[3], t.sn.v[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t x = a.v[j], y = b.v[j];
            a.v[j] = f32x2_fma(x, t.cs.v[j], f32x2_mul(y, negated(t.sn.v[j])));
            b.v[j] = f32x2_fma(x, t.sn.v[j], f32x2_mul(y, t.cs.v[j]));
        }
    }
}

template <int LANES_LOG2>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = 1; o < (1 << LANES_LOG2); o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// sum over the lane's 16 elements of x * y
__device__ __forceinline__ float dot16(const Pairs& xa, const Pairs& xb, const Pairs& ya, const Pairs& yb) {
    uint64_t s = f32x2_mul(xa.v[0], ya.v[0]), t = f32x2_mul(xb.v[0], yb.v[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) {
        s = f32x2_fma(xa.v[j], ya.v[j], s);
        t = f32x2_fma(xb.v[j], yb.v[j], t);
    }
    float u, v;
    f32x2_split(f32x2_add(s, t), u, v);
    return u + v;
}

template <bool NORM>
__device__ __forceinline__ void load_factors(const QkArgs& p, Shared& sm) {
    const float add = (p.flags & RAPID_QK_UNIT_OFFSET) ? 1.f : 0.f;
    const int i = threadIdx.x;
    static_assert(kThreads >= kMaxHeadDim, "one element a thread");
    if (NORM && i < p.head_dim) {
        sm.weight[0][i] = p.q_weight[i] + add;
        sm.weight[1][i] = p.k_weight[i] + add;
    }
    if (i < p.rot_dim / 2) sm.turns[i] = (double)p.inv_freq[i] * 0.15915494309189533577;  // turns a position: 1 / (2 pi)
    __syncthreads();
}

// a lane's part of a row's head that has nothing in it
template <class T>
__device__ __forceinline__ void store_zeros(T* dst, const Place& x) {
    const float z[8] = {};
    Vec8<T>::store(dst + x.a, z);
    Vec8<T>::store(dst + x.b, z);
}

template <class T, int LANES_LOG2, bool INTER, bool NORM>
__global__ void __launch_bounds__(kThreads, 2)
qk_fwd_kernel(QkArgs p, const T* q, const T* k, T* q_out, T* k_out) {
    __shared__ __align__(16) Shared sm;
    constexpr int lanes = 1 << LANES_LOG2, groups = kThreads >> LANES_LOG2;
    const int group = threadIdx.x >> LANES_LOG2;
    const int per_row = p.per_row, rows = groups / per_row;
    const int row = group / per_row, h0 = group - row * per_row;
    const Place x = place_of(p, threadIdx.x & (lanes - 1));
    load_factors<NORM>(p, sm);
    const WarpRows mine_rows = warp_rows<LANES_LOG2>(per_row);
    const int angle_at = (row - mine_rows.first) * (p.rot_dim / 2) + x.angle;
    const float *cs_at = sm.cs[threadIdx.x >> 5] + angle_at, *sn_at = sm.sn[threadIdx.x >> 5] + angle_at;
    const int b_after_a = INTER ? 8 : x.b - x.a;
    Vec8<T> va[kAhead<T>] = {}, vb[kAhead<T>] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < p.n_rows; r0 += (int64_t)gridDim.x * rows) {
        const int64_t r = r0 + row;
        const bool have = row < rows && r < p.n_rows && x.on, live = have && row_live(p, r);
        const bool warp_live = __any_sync(0xffffffffu, live);
        if (!warp_live) {  // nothing but masked rows
            for (int h = h0; have && h < p.heads; h += per_row)
                store_zeros(h < p.heads_q ? q_out + r * p.ld_q_out + h * p.head_dim : k_out + r * p.ld_k_out + (h - p.heads_q) * p.head_dim, x);
            continue;
        }
        const double pos = position(p, r0 + mine_rows.first + (threadIdx.x & 31));
        const T *qr = q + r * p.ld_q + x.a, *kr = k + r * p.ld_k + x.a - (int64_t)p.heads_q * p.head_dim;
        T *qo = q_out + r * p.ld_q_out + x.a, *ko = k_out + r * p.ld_k_out + x.a - (int64_t)p.heads_q * p.head_dim;
        bool angled = false;
        Angles<INTER> turns;
        // the same number of turns in every lane: the sums exchange over whole warps
#pragma unroll 1
        for (int h1 = h0; h1 - h0 < p.heads; h1 += kAhead<T> * per_row) {
#pragma unroll
            for (int i = 0; i < kAhead<T>; ++i) {
                const int h = h1 + i * per_row;
                if (live && h < p.heads) {
                    const T* src = (h < p.heads_q ? qr : kr) + h * p.head_dim;
                    va[i].load(src);
                    vb[i].load(src + b_after_a);
                }
            }
            if (!angled) {
                __syncwarp();  // the last rows' angles have been read
                angles(p, sm, mine_rows.count, pos);
                __syncwarp();
                if (x.angle >= 0) turns.from(cs_at, sn_at, false);
                angled = true;
            }
#pragma unroll
            for (int i = 0; i < kAhead<T>; ++i) {
                const int h = h1 + i * per_row;
                if (h - h0 >= p.heads) break;  // the same for all lanes
                // heads and rows that a group does not have run along with whatever its registers hold
                Pairs a, b;
                a.from(va[i]);
                b.from(vb[i]);
                if (NORM) {
                    const float own = dot16(a, b, a, b), sq = group_sum<LANES_LOG2>(x.on ? own : 0.f);
                    const float rstd = rsqrtf(sq * p.inv_dim + p.eps);
                    const float* w = sm.weight[h < p.heads_q ? 0 : 1];
                    Pairs wa, wb;
                    wa.from(w + x.a);
                    wb.from(w + x.b);
                    a.times(wa);
                    b.times(wb);
                    a.times(rstd);
                    b.times(rstd);
                }
                if (x.angle >= 0) rotate<INTER>(a, b, turns);
                if (have && h < p.heads) {
                    T* dst = (h < p.heads_q ? qo : ko) + h * p.head_dim;
                    if (live) {
                        a.store(dst);
                        b.store(dst + b_after_a);
                    } else {
                        store_zeros(dst - x.a, x);
                    }
                }
            }
        }
    }
}

// The gradient of the queries (blocks [0, blocks_q)) and of the keys (the others); `first`, `blocks` and per_row are of the
// block's kind.  A lane keeps its 16 sums of the weight gradient in registers; a block adds its groups in order at the end
// and leaves one partial sum, which qk_weight_grad_kernel adds in order.
struct QkBwdKind {
    const void *in, *gout;
    void* gin;
    int64_t ld_in, ld_gout, ld_gin;
    int heads, per_row, first, blocks;
};
struct QkBwdKinds {
    QkBwdKind kind[2];
};

template <class T, int LANES_LOG2, bool INTER, bool NORM>
__global__ void __launch_bounds__(kThreads, 2)
qk_bwd_kernel(QkArgs p, QkBwdKinds both, float* __restrict__ partial) {
    constexpr int kTurn = sizeof(T) == 2 ? 2 : 1;  // heads of a group in flight, each of two matrices
    __shared__ __align__(16) Shared sm;
    __shared__ float part[kThreads][17];
    constexpr int lanes = 1 << LANES_LOG2, groups = kThreads >> LANES_LOG2;
    const int which = (int)blockIdx.x < both.kind[0].blocks ? 0 : 1;
    const QkBwdKind m = which ? both.kind[1] : both.kind[0];
    const int heads = m.heads, per_row = m.per_row;
    const int group = threadIdx.x >> LANES_LOG2;
    const int rows = groups / per_row, row = group / per_row, h0 = group - row * per_row;
    const Place x = place_of(p, threadIdx.x & (lanes - 1));
    load_factors<NORM>(p, sm);
    const WarpRows mine_rows = warp_rows<LANES_LOG2>(per_row);
    const int angle_at = (row - mine_rows.first) * (p.rot_dim / 2) + x.angle;
    const float *cs_at = sm.cs[threadIdx.x >> 5] + angle_at, *sn_at = sm.sn[threadIdx.x >> 5] + angle_at;
    const float *wa_at = sm.weight[which] + x.a, *wb_at = sm.weight[which] + x.b;
    const int b_after_a = INTER ? 8 : x.b - x.a;
    Vec8<T> xa[kTurn] = {}, xb[kTurn] = {}, ya[kTurn] = {}, yb[kTurn] = {};
    Pairs dwa, dwb;
    dwa.zero();
    dwb.zero();
    for (int64_t r0 = (int64_t)((int)blockIdx.x - m.first) * rows; r0 < p.n_rows; r0 += (int64_t)m.blocks * rows) {
        const int64_t r = r0 + row;
        const bool have = row < rows && r < p.n_rows && x.on, live = have && row_live(p, r);
        const T* in = static_cast<const T*>(m.in) + r * m.ld_in + x.a;
        const T* gout = static_cast<const T*>(m.gout) + r * m.ld_gout + x.a;
        T* gin = static_cast<T*>(m.gin) + r * m.ld_gin + x.a;
        if (!__any_sync(0xffffffffu, live)) {  // nothing but masked rows
            for (int h = h0; have && h < heads; h += per_row) store_zeros(gin - x.a + h * p.head_dim, x);
            continue;
        }
        const double pos = position(p, r0 + mine_rows.first + (threadIdx.x & 31));
        bool angled = false;
#pragma unroll 1
        for (int h1 = h0; h1 - h0 < heads; h1 += kTurn * per_row) {
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                const int h = h1 + i * per_row;
                if (live && h < heads) {
                    if (NORM) {
                        xa[i].load(in + h * p.head_dim);
                        xb[i].load(in + h * p.head_dim + b_after_a);
                    }
                    ya[i].load(gout + h * p.head_dim);
                    yb[i].load(gout + h * p.head_dim + b_after_a);
                }
            }
            if (!angled) {
                __syncwarp();  // the last rows' angles have been read
                angles(p, sm, mine_rows.count, pos);
                __syncwarp();
                angled = true;
            }
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                const int h = h1 + i * per_row;
                if (h - h0 >= heads) break;  // the same for all lanes
                // heads and rows that a group does not have run along with whatever its registers hold
                const bool mine = have && h < heads;
                asm volatile("" ::: "memory");  // one head after the other: together they do not fit the registers
                Pairs a, b, ga, gb;
                ga.from(ya[i]);
                gb.from(yb[i]);
                if (x.angle >= 0) {
                    Angles<INTER> turns;
                    turns.from(cs_at, sn_at, true);
                    rotate<INTER>(ga, gb, turns);
                }
                if constexpr (NORM) {
                    a.from(xa[i]);
                    b.from(xb[i]);
                    // both sums go round together: x . x, and (w y') . x, of which xh = x * rstd needs rstd more
                    Pairs wa, wb;
                    wa.from(wa_at);
                    wb.from(wb_at);
                    wa.times(ga);
                    wb.times(gb);
                    float sq = dot16(a, b, a, b), dot = dot16(wa, wb, a, b);
                    if (!x.on) sq = dot = 0.f;
#pragma unroll
                    for (int o = 1; o < lanes; o <<= 1) {
                        sq += __shfl_xor_sync(0xffffffffu, sq, o);
                        dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    }
                    if (live && mine) {
                        const float rstd = rsqrtf(sq * p.inv_dim + p.eps);
                        // dx = rstd (w y' - xh mean(w y' xh)) = rstd w y' - x rstd^3 (w y' . x) / head_dim
                        const float back = -dot * p.inv_dim * rstd * rstd * rstd;
                        const uint64_t r2 = f32x2(rstd, rstd), b2 = f32x2(back, back);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            dwa.v[j] = f32x2_fma(ga.v[j], f32x2_mul(a.v[j], r2), dwa.v[j]);
                            dwb.v[j] = f32x2_fma(gb.v[j], f32x2_mul(b.v[j], r2), dwb.v[j]);
                            ga.v[j] = f32x2_fma(a.v[j], b2, f32x2_mul(wa.v[j], r2));
                            gb.v[j] = f32x2_fma(b.v[j], b2, f32x2_mul(wb.v[j], r2));
                        }
                    }
                }
                if (mine) {
                    T* dst = gin + h * p.head_dim;
                    if (live) {
                        ga.store(dst);
                        gb.store(dst + b_after_a);
                    } else {
                        store_zeros(dst - x.a, x);
                    }
                }
            }
        }
    }
    if constexpr (NORM) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x2_split(dwa.v[j], part[threadIdx.x][2 * j], part[threadIdx.x][2 * j + 1]);
            f32x2_split(dwb.v[j], part[threadIdx.x][8 + 2 * j], part[threadIdx.x][9 + 2 * j]);
        }
        __syncthreads();
        // thread (lane u of a group, element j): the sum over the block's groups
        for (int i = threadIdx.x; i < lanes * 16; i += kThreads) {
            const int u = i >> 4, j = i & 15;
            const Place y = place_of(p, u);
            if (!y.on) continue;
            float sum = 0.f;
            for (int g = 0; g < groups; ++g) sum += part[g * lanes + u][j];
            partial[(size_t)blockIdx.x * kMaxHeadDim + (j < 8 ? y.a + j : y.b + j - 8)] = sum;
        }
    }
}

// One block for each kind and 8 columns: 32 threads a column each add every 32nd partial sum, then the 32 sums in order.
__global__ void __launch_bounds__(256)
qk_weight_grad_kernel(int blocks_q, int blocks_k, const float* __restrict__ partial, float* __restrict__ dq_weight,
                      float* __restrict__ dk_weight) {
    __shared__ double part[8][33];
    const int kind = blockIdx.y, col = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int c = blockIdx.x * 8 + col;
    const int from = kind ? blocks_q : 0, to = kind ? blocks_q + blocks_k : blocks_q;
    double sum = 0.0;
#pragma unroll 4
    for (int b = from + slice; b < to; b += 32) sum += (double)partial[(size_t)b * kMaxHeadDim + c];
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
    // far beyond any device's memory; keeps every size below in 64 bits
    const int64_t rows = (int64_t)d->n_seq * d->seq_len, most = (1ll << 56) / rows < (1ll << 31) ? (1ll << 56) / rows : 1ll << 31;
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
                 const int32_t* positions, const uint8_t* mask) {
    QkArgs p{};
    p.n_rows = (int64_t)d.n_seq * d.seq_len;
    p.seq_len = d.seq_len;
    p.heads_q = d.n_q_heads;
    p.heads = d.n_q_heads + d.n_k_heads;
    p.head_dim = d.head_dim;
    p.rot_dim = d.rot_dim;
    p.lanes_log2 = d.head_dim <= 64 ? 2 : d.head_dim <= 128 ? 3 : 4;
    p.flags = d.flags;
    p.eps = d.eps;
    p.inv_dim = 1.f / (float)d.head_dim;
    p.ld_q = d.ld_q;
    p.ld_k = d.ld_k;
    p.ld_q_out = d.ld_q_out;
    p.ld_k_out = d.ld_k_out;
    p.q_weight = q_weight;
    p.k_weight = k_weight;
    p.inv_freq = inv_freq;
    p.positions = positions;
    p.mask = mask;
    return p;
}

// Groups on one row, so that each has up to `ahead` heads to take; with few rows more, for about `blocks` blocks.
int groups_per_row(const QkArgs& p, int heads, int ahead, int64_t blocks) {
    const int groups = kThreads >> p.lanes_log2, most = heads < groups ? heads : groups;
    int per_row = (heads + ahead - 1) / ahead;
    while (per_row < most && p.n_rows * per_row < blocks * groups) per_row *= 2;
    return per_row < most ? per_row : most;
}
int tile_rows(const QkArgs& p, int per_row) { return (kThreads >> p.lanes_log2) / per_row; }

template <class T, int LANES_LOG2>
void run_fwd_as(const QkArgs& p, unsigned grid, const T* q, const T* k, T* q_out, T* k_out, cudaStream_t st) {
    const bool inter = (p.flags & RAPID_QK_INTERLEAVED) != 0, norm = !(p.flags & RAPID_QK_NO_NORM);
    auto kern = inter ? (norm ? qk_fwd_kernel<T, LANES_LOG2, true, true> : qk_fwd_kernel<T, LANES_LOG2, true, false>)
                      : (norm ? qk_fwd_kernel<T, LANES_LOG2, false, true> : qk_fwd_kernel<T, LANES_LOG2, false, false>);
    kern<<<grid, kThreads, 0, st>>>(p, q, k, q_out, k_out);
}
template <class T>
void run_fwd(const QkArgs& p, unsigned grid, const void* q, const void* k, void* q_out, void* k_out, cudaStream_t st) {
    auto run = p.lanes_log2 == 2 ? run_fwd_as<T, 2> : p.lanes_log2 == 3 ? run_fwd_as<T, 3> : run_fwd_as<T, 4>;
    run(p, grid, static_cast<const T*>(q), static_cast<const T*>(k), static_cast<T*>(q_out), static_cast<T*>(k_out), st);
}

template <class T, int LANES_LOG2>
void run_bwd_as(const QkArgs& p, const QkBwdKinds& both, float* partial, cudaStream_t st) {
    const bool inter = (p.flags & RAPID_QK_INTERLEAVED) != 0, norm = !(p.flags & RAPID_QK_NO_NORM);
    auto kern = inter ? (norm ? qk_bwd_kernel<T, LANES_LOG2, true, true> : qk_bwd_kernel<T, LANES_LOG2, true, false>)
                      : (norm ? qk_bwd_kernel<T, LANES_LOG2, false, true> : qk_bwd_kernel<T, LANES_LOG2, false, false>);
    kern<<<(unsigned)(both.kind[0].blocks + both.kind[1].blocks), kThreads, 0, st>>>(p, both, partial);
}
template <class T>
void run_bwd(const QkArgs& p, const QkBwdKinds& both, float* partial, cudaStream_t st) {
    auto run = p.lanes_log2 == 2 ? run_bwd_as<T, 2> : p.lanes_log2 == 3 ? run_bwd_as<T, 3> : run_bwd_as<T, 4>;
    run(p, both, partial, st);
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
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(inv_freq, 4) || !aligned(positions, 4))
        return RAPID_ERR_ALIGNMENT;
    if (!(d.flags & RAPID_QK_NO_NORM) && (!aligned(q_weight, 4) || !aligned(k_weight, 4))) return RAPID_ERR_ALIGNMENT;
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
    QkArgs p = make_args(d, q_weight, k_weight, inv_freq, positions, mask);
    p.per_row = groups_per_row(p, p.heads, d.dtype == RAPID_BF16 ? kAhead<uint16_t> : kAhead<float>, 2 * sms);
    const int64_t rows = tile_rows(p, p.per_row), tiles = (p.n_rows + rows - 1) / rows;
    const unsigned grid = (unsigned)(tiles < 2 * sms ? tiles : 2 * sms);  // two blocks are resident on an SM
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d.dtype == RAPID_BF16) run_fwd<uint16_t>(p, grid, q, k, q_out, k_out, st);
    else run_fwd<float>(p, grid, q, k, q_out, k_out, st);
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}

extern "C" rapid_status_t rapid_qk_norm_rope_bwd_workspace_bytes(const rapid_qk_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    rapid_status_t s = check_qk(desc, true);
    if (s != RAPID_OK) return s;
    *bytes = (size_t)kMaxBwdBlocks * kMaxHeadDim * sizeof(float);
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
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(dq_out, 16) || !aligned(dk_out, 16) || !aligned(dq, 16) || !aligned(dk, 16) ||
        !aligned(inv_freq, 4) || !aligned(positions, 4))
        return RAPID_ERR_ALIGNMENT;
    if (norm && (!aligned(q_weight, 4) || !aligned(k_weight, 4) || !aligned(dq_weight, 4) || !aligned(dk_weight, 4))) return RAPID_ERR_ALIGNMENT;
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
    QkArgs p = make_args(d, q_weight, k_weight, inv_freq, positions, mask);
    const int most = 2 * sms < kMaxBwdBlocks ? 2 * sms : kMaxBwdBlocks;  // two blocks are resident on an SM
    QkBwdKinds both = {{{q, dq_out, dq, d.ld_q, d.ld_q_out, d.ld_dq, d.n_q_heads, 1, 0, 0}, {k, dk_out, dk, d.ld_k, d.ld_k_out, d.ld_dk, d.n_k_heads, 1, 0, 0}}};
    // Blocks in proportion to the heads, a row's angles counted as two heads more (one: 124 us, three: 127, two: 120, 64 x 1024).
    int share = (int)((int64_t)most * (d.n_k_heads + 2) / (p.heads + 4));
    share = share < 1 ? 1 : share;
    for (int i = 0; i < 2; ++i) {
        QkBwdKind& m = both.kind[i];
        const int64_t room = i ? share : most - share;
        m.per_row = groups_per_row(p, m.heads, 6, room);
        const int64_t rows = tile_rows(p, m.per_row), tiles = (p.n_rows + rows - 1) / rows;
        m.blocks = (int)(tiles < room ? tiles : room);
    }
    both.kind[1].first = both.kind[0].blocks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float* partial = static_cast<float*>(workspace);
    if (d.dtype == RAPID_BF16) run_bwd<uint16_t>(p, both, partial, st);
    else run_bwd<float>(p, both, partial, st);
    if (norm)
        qk_weight_grad_kernel<<<dim3((unsigned)(d.head_dim / 8), 2), 256, 0, st>>>(both.kind[0].blocks, both.kind[1].blocks, partial,
                                                                                 dq_weight, dk_weight);
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}
