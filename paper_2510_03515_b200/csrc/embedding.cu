// Token embedding with scaling, and its gradient over sorted tokens.  Both are bound by HBM bytes.
//
// Forward: a warp copies up to 2048 columns of one row (8 vectors of 8 elements a lane, all loads in flight before the first
// store), times the scale.
//
// Gradient: dtable[v] = s * sum of the rows of dout whose token is v.  No float atomics: the row numbers are sorted by
// token with a stable radix sort (9-bit digits, written here), so a token's rows lie next to each other in row order, and
// every sum has a fixed order.  Frequent tokens (a few per cent of all rows each) would keep one warp busy for long, so any
// 32 sorted positions [32 j, 32 j + 32) that hold one token are summed first, by a warp of their own; a row of dtable
// is then at most 31 rows + the pieces + 31 rows.  The last kernel writes dtable: most of its rows belong to tokens that do
// not occur, and one warp of each block writes those as bulk copies of zeros out of shared memory, which needs no registers
// and hardly an instruction, while the other warps sum.
//
// Measured: 64 x 1024 tokens x 1536 bf16, over a third of them masked: forward 43 us (5.7 TB/s).  Gradient into 151936 rows of float:
// 434 us with a warp a token and segment, 299 with the radix sort's wide digits, 248 with frequent tokens summed by blocks and
// the others a whole row at a time, 244 with the sort's loads issued ahead, 240 (4.4 TB/s) now; its last kernel takes 200 of
// them, the sort and the lists before it the rest.  Into bf16 170, added to a table 154, 256 x 1024 rows of 512 172, 64 x 1024 of
// 2048 into 128256 276.  16384 rows of 512 into 32000: 92 us, 53 with the sort over several blocks and narrow rows eight at a time.
// The last kernel holds 48 sums and two rows of 24 registers in the 128 that two blocks an SM leave a thread: it spills 24 of them
// (bf16 rows; 10 with float rows).
#include <math.h>

#include "policy_ops.cuh"
#include "tma_pipe.cuh"

namespace rapid {
namespace policy {
namespace {

constexpr int kSegVecs = 8;                 // forward: vectors of 8 elements a lane takes of a row
constexpr int kFwdSeg = kSegVecs * 32 * 8;  // columns a warp takes of a row

template <class T>
__global__ void __launch_bounds__(256)
embed_fwd_kernel(int64_t n_rows, int segs, int vocab, int dim, int64_t ld_table, int64_t ld_out, float scale,
                 const int32_t* __restrict__ tokens, const uint8_t* __restrict__ mask, const T* __restrict__ table,
                 T* __restrict__ out, rapid_stats_t* stats) {
    __shared__ int counts[2];
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (stats) {
        if (threadIdx.x < 2) counts[threadIdx.x] = 0;
        __syncthreads();
    }
    if (unit < n_rows * segs) {
        const int64_t r = unit / segs;
        const int seg = (int)(unit - r * segs);
        const int tok = tokens[r];
        const bool live = mask == nullptr || mask[r] != 0;
        const bool ok = live && tok >= 0 && tok < vocab;
        if (stats && seg == 0 && lane == 0 && live) atomicAdd(&counts[ok ? 0 : 1], 1);
        const T* src = table + (ok ? (int64_t)tok * ld_table : 0);
        T* dst = out + r * ld_out;
        const int c0 = seg * kFwdSeg + lane * 8;
        Vec8<T> v[kSegVecs];
        if (ok) {
#pragma unroll
            for (int i = 0; i < kSegVecs; ++i)
                if (c0 + i * 256 + 8 <= dim) v[i].load(src + c0 + i * 256);
        }
#pragma unroll
        for (int i = 0; i < kSegVecs; ++i) {
            const int c = c0 + i * 256;
            if (c + 8 <= dim) {
                float f[8];
                v[i].get(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = ok ? f[j] * scale : 0.f;
                Vec8<T>::store(dst + c, f);
            } else {  // the row's ragged end
                for (int j = c; j < dim; ++j) from_float(dst + j, ok ? to_float(src[j]) * scale : 0.f);
            }
        }
    }
    if (stats) {
        __syncthreads();
        if (threadIdx.x == 0 && counts[0]) atomicAdd(reinterpret_cast<unsigned long long*>(&stats->n_tokens), (unsigned long long)counts[0]);
        if (threadIdx.x == 0 && counts[1]) atomicAdd(&stats->n_bad_token, counts[1]);
    }
}

// ---- stable radix sort of (token, row) ----------------------------------------------------------------------

constexpr int kRadixBits = 9, kBins = 1 << kRadixBits;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;  // one thread a digit value
constexpr int kMaxSortBlocks = 64;  // every block reads the histograms of all
constexpr int kMinSortRows = 1024;
constexpr int kSortAhead = 8;
// Up to here one block sorts alone, without histograms and launches in between (151936 tokens, one block against several:
// 2000 rows 9.3 and 9.4 us, 4000 13.6 and 15.4, 6000 19.3 and 16.1, 16000 44 and 15).
constexpr int64_t kOneBlockRows = 5120;

// The rows of block b are [b * per_block, (b + 1) * per_block); within it warp w has a run of per_block / 16 of them.
struct SortShape {
    int64_t n_rows, per_block;
    int blocks, passes;
};

inline SortShape sort_shape(int64_t n_rows, int32_t vocab) {
    SortShape s;
    s.n_rows = n_rows;
    // one block does not need the histograms of others and finishes in one launch
    const int64_t want = n_rows <= kOneBlockRows ? 1 : (n_rows + kMinSortRows - 1) / kMinSortRows;
    s.blocks = (int)(want < kMaxSortBlocks ? want : kMaxSortBlocks);
    s.per_block = (n_rows + s.blocks - 1) / s.blocks;
    s.per_block = (s.per_block + kSortThreads - 1) / kSortThreads * kSortThreads;  // whole warps' runs
    s.blocks = (int)((n_rows + s.per_block - 1) / s.per_block);
    int bits = 0;
    while ((1ll << bits) <= (int64_t)vocab) ++bits;  // keys 0 .. vocab; `vocab` marks rows that do not count
    s.passes = (bits + kRadixBits - 1) / kRadixBits;
    return s;
}

struct SortArgs {
    const int32_t* tokens;
    const uint8_t* mask;
    int vocab;
    const uint32_t* key_in;  // nullptr in the first pass: keys come from the tokens
    const uint32_t* row_in;
    uint32_t* key_out;
    uint32_t* row_out;
    uint32_t* hist;  // [blocks][kBins]
    uint32_t* used;  // counters of the tokens that occur, cleared by the first launch
    int shift;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t i) {
    if (a.key_in) return a.key_in[i];
    const int tok = a.tokens[i];
    const bool ok = (a.mask == nullptr || a.mask[i] != 0) && tok >= 0 && tok < a.vocab;
    return ok ? (uint32_t)tok : (uint32_t)a.vocab;
}

__global__ void __launch_bounds__(kSortThreads) sort_hist_kernel(SortArgs a, SortShape s) {
    __shared__ uint32_t bins[kBins];
    if (blockIdx.x == 0 && threadIdx.x < 2) a.used[threadIdx.x] = 0;
    bins[threadIdx.x] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * s.per_block, hi = min(lo + s.per_block, s.n_rows);
    for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&bins[(sort_key(a, i) >> a.shift) & (kBins - 1)], 1u);
    __syncthreads();
    a.hist[(size_t)blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

// One pass of one block.  `alone`: the block holds all rows, its own counts are the totals.
__device__ __forceinline__ void sort_scatter(const SortArgs& a, const SortShape& s, bool alone, uint32_t (*cnt)[kBins],
                                             uint32_t* scan) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int i = tid; i < kSortWarps * kBins; i += kSortThreads) (&cnt[0][0])[i] = 0;
    __syncthreads();
    const int64_t run = s.per_block / kSortWarps;  // a multiple of 32
    const int64_t lo = (int64_t)blockIdx.x * s.per_block + warp * run, hi = min(lo + run, s.n_rows);
    // kSortAhead turns of 32 rows are loaded before the first is used
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kSortAhead) {
        uint32_t key[kSortAhead];
#pragma unroll
        for (int t = 0; t < kSortAhead; ++t) key[t] = i0 + 32 * t + lane < hi ? sort_key(a, i0 + 32 * t + lane) : 0u;
#pragma unroll
        for (int t = 0; t < kSortAhead; ++t)
            if (i0 + 32 * t + lane < hi) atomicAdd(&cnt[warp][(key[t] >> a.shift) & (kBins - 1)], 1u);
    }
    // this thread's digit: how many rows lie in blocks before this one, and how many in all
    uint32_t before = 0, total = 0;
    if (!alone) {
#pragma unroll 16
        for (int b = 0; b < s.blocks; ++b) {
            const uint32_t h = a.hist[(size_t)b * kBins + tid];
            total += h;
            before += b < (int)blockIdx.x ? h : 0u;
        }
    }
    __syncthreads();
    if (alone) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) total += cnt[w][tid];
    }
    // exclusive sum of the totals over the digits
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    uint32_t base = incl - total + before;
    for (int w = 0; w < warp; ++w) base += scan[w];
    // first place of each warp's rows of this digit
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = cnt[w][tid];
        cnt[w][tid] = base;
        base += c;
    }
    __syncthreads();
    // in row order, 32 rows at a time: a row's place is the digit's next one plus the equal digits in lower lanes
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kSortAhead) {
        uint32_t key[kSortAhead], row[kSortAhead];
#pragma unroll
        for (int t = 0; t < kSortAhead; ++t) {
            const int64_t i = i0 + 32 * t + lane;
            key[t] = i < hi ? sort_key(a, i) : 0u;
            row[t] = i < hi && a.row_in ? a.row_in[i] : (uint32_t)i;
        }
#pragma unroll
        for (int t = 0; t < kSortAhead; ++t) {
            if (i0 + 32 * t >= hi) break;
            const bool on = i0 + 32 * t + lane < hi;
            const uint32_t digit = on ? (key[t] >> a.shift) & (kBins - 1) : (uint32_t)kBins;
            const unsigned peers = __match_any_sync(0xffffffffu, digit);
            const int first = __ffs(peers) - 1;
            uint32_t place = 0;
            if (on && lane == first) {
                place = cnt[warp][digit];
                cnt[warp][digit] = place + __popc(peers);
            }
            place = __shfl_sync(0xffffffffu, place, first) + __popc(peers & ((1u << lane) - 1u));
            if (on) {
                a.key_out[place] = key[t];
                a.row_out[place] = row[t];
            }
            __syncwarp();
        }
    }
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(SortArgs a, SortShape s) {
    __shared__ uint32_t cnt[kSortWarps][kBins];
    __shared__ uint32_t scan[kSortWarps];
    sort_scatter(a, s, false, cnt, scan);
}

// All passes of a sort that fits one block.  Ends in (key_b, row_b) after an even number of passes, (key_a, row_a) after an
// odd one, like the multi-block form.
__global__ void __launch_bounds__(kSortThreads)
sort_one_block_kernel(SortArgs a, SortShape s, uint32_t* key_a, uint32_t* row_a, uint32_t* key_b, uint32_t* row_b) {
    __shared__ uint32_t cnt[kSortWarps][kBins];
    __shared__ uint32_t scan[kSortWarps];
    if (threadIdx.x < 2) a.used[threadIdx.x] = 0;
    for (int p = 0; p < s.passes; ++p) {
        a.shift = p * kRadixBits;
        a.key_in = p == 0 ? nullptr : (p & 1) ? key_a : key_b;
        a.row_in = p == 0 ? nullptr : (p & 1) ? row_a : row_b;
        a.key_out = (p & 1) ? key_b : key_a;
        a.row_out = (p & 1) ? row_b : row_a;
        sort_scatter(a, s, true, cnt, scan);
        __syncthreads();  // the block's own writes are its next pass's inputs
    }
}

// ---- sums over a token's rows -------------------------------------------------------------------------------

constexpr int kPiece = 32;  // sorted positions of a piece

// A warp sums K vectors of 8 columns a lane, 256 K columns, with kAhead rows of dout in flight.  Most tokens occur once or
// twice: what is in flight is then the width, so their rows are taken whole (WIDE).  Frequent tokens take a narrower segment
// with more rows in flight.
template <class T, bool WIDE>
struct Seg {
    static constexpr int K = (WIDE ? 6 : 2) / (sizeof(T) == 2 ? 1 : 2);
    static constexpr int kAhead = WIDE ? 2 : 8;
    static constexpr int kColumns = K * 256;
};
constexpr uint32_t kFrequent = 8;  // tokens that occur more often are summed by a whole block

// acc += rows of dout at sorted positions [lo, hi), in order
template <class T, bool WIDE>
__device__ __forceinline__ void add_rows(float (&acc)[Seg<T, WIDE>::K][8], const uint32_t* __restrict__ rows, int64_t lo, int64_t hi,
                                         const T* __restrict__ dout, int64_t ld, int c0, int dim, int lane) {
    constexpr int K = Seg<T, WIDE>::K, kAhead = Seg<T, WIDE>::kAhead;
    for (int64_t i0 = lo; i0 < hi; i0 += 32) {
        const int n = (int)min((int64_t)32, hi - i0);
        const uint32_t mine = lane < n ? rows[i0 + lane] : 0u;
        for (int i = 0; i < n; i += kAhead) {
            Vec8<T> v[kAhead][K];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const T* src = dout + (int64_t)__shfl_sync(0xffffffffu, mine, min(i + u, n - 1)) * ld;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int c = c0 + k * 256;
                    if (i + u < n && c + 8 <= dim) v[u][k].load(src + c);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const T* src = dout + (int64_t)__shfl_sync(0xffffffffu, mine, min(i + u, n - 1)) * ld;
                if (i + u < n) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const int c = c0 + k * 256;
                        if (c + 8 <= dim) {
                            float f[8];
                            v[u][k].get(f);
#pragma unroll
                            for (int j = 0; j < 8; ++j) acc[k][j] += f[j];
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (c + j < dim) acc[k][j] += to_float(src[c + j]);
                        }
                    }
                }
            }
        }
    }
}

// A token that occurs: its rows are at sorted positions [lo, hi).
struct __align__(16) Used {
    uint32_t token, lo, hi, pad;
};

struct GradArgs {
    int64_t n_rows;
    int segs, wide_segs, dim, vocab;  // segments of a row for frequent tokens (and pieces), for the others
    int64_t ld, ldp, ld_table;
    float scale;
    bool accumulate;
    const uint32_t *keys, *rows;
    uint32_t* start;  // [vocab + 1]: first sorted position of each token
    uint32_t* used;   // how many tokens occur seldom, how many often
    Used* list;       // which, in any order: the former from the front, the latter from the back
    uint32_t room;    // of the list
    float* pieces;    // [n_rows / kPiece][ldp]
};

__device__ __forceinline__ uint32_t lower_bound(const uint32_t* __restrict__ keys, uint32_t n, uint32_t v) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = lo + ((hi - lo) >> 1);
        if (keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

constexpr int kTokensPerBlock = 1024;

// Blocks [0, token_blocks): where each token's rows begin, and the list of the tokens that occur.  The others: sums of whole
// pieces, a warp for each piece and segment.
template <class T>
__global__ void __launch_bounds__(256) embed_prepare_kernel(GradArgs a, int token_blocks, const T* __restrict__ dout) {
    constexpr int K = Seg<T, false>::K;
    const int lane = threadIdx.x & 31;
    if ((int)blockIdx.x < token_blocks) {
        __shared__ uint32_t first[kTokensPerBlock + 1];
        const uint32_t v0 = blockIdx.x * (uint32_t)kTokensPerBlock, n = (uint32_t)a.n_rows;
        // four searches of a thread side by side: each step is one trip to L2
        uint32_t lo[4] = {0, 0, 0, 0}, hi[4] = {n, n, n, n};
        for (uint32_t width = n; width > 0; width >>= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lo[i] < hi[i]) {
                    const uint32_t mid = lo[i] + ((hi[i] - lo[i]) >> 1);
                    if (a.keys[mid] < v0 + threadIdx.x + 256u * i) lo[i] = mid + 1;
                    else hi[i] = mid;
                }
#pragma unroll
        for (int i = 0; i < 4; ++i) first[threadIdx.x + 256 * i] = lo[i];
        if (threadIdx.x == 0) first[kTokensPerBlock] = lower_bound(a.keys, n, v0 + kTokensPerBlock);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at_v = threadIdx.x + 256u * i, v = v0 + at_v;
            const uint32_t from = first[at_v], to = first[at_v + 1];
            if (v <= (uint32_t)a.vocab) a.start[v] = from;
            const uint32_t count = v < (uint32_t)a.vocab ? to - from : 0u;
#pragma unroll
            for (int often = 0; often < 2; ++often) {
                const bool mine = often ? count > kFrequent : count > 0 && count <= kFrequent;
                const unsigned which = __ballot_sync(0xffffffffu, mine);
                uint32_t at = 0;
                if (lane == 0 && which) at = atomicAdd(a.used + often, (uint32_t)__popc(which));
                at = __shfl_sync(0xffffffffu, at, 0) + __popc(which & ((1u << lane) - 1u));
                if (mine) a.list[often ? a.room - 1u - at : at] = Used{v, from, to, 0u};
            }
        }
        return;
    }
    const int64_t unit = (int64_t)(blockIdx.x - token_blocks) * 8 + (threadIdx.x >> 5);
    const int64_t piece = unit / a.segs;
    const int64_t lo = piece * kPiece, hi = lo + kPiece;
    if (hi > a.n_rows) return;  // whole pieces only
    const uint32_t key = a.keys[lo];
    if (key != a.keys[hi - 1] || key >= (uint32_t)a.vocab) return;
    const int c0 = (int)(unit - piece * a.segs) * (K * 256) + lane * 8;
    float acc[K][8] = {};
    add_rows<T, false>(acc, a.rows, lo, hi, dout, a.ld, c0, a.dim, lane);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (c0 + k * 256 < a.dim) Vec8<float>::store(a.pieces + piece * a.ldp + c0 + k * 256, acc[k]);
}

constexpr int kZeroBytes = 8192;

// Warp 7 of a block: rows of dtable whose token does not occur, the rows of tokens [from, to).
template <class G>
__device__ __forceinline__ void write_zeros(const GradArgs& a, uint8_t* zeros, int64_t from, int64_t to, G* __restrict__ dtable, int lane) {
    for (int i = lane; i < kZeroBytes / 16; i += 32) reinterpret_cast<uint4*>(zeros)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncwarp();
    const uint32_t bytes = (uint32_t)((int64_t)a.dim * sizeof(G) / 16 * 16);  // the rest of a row is less than a vector
    for (int64_t v0 = from; v0 < to; v0 += 32) {
        const int64_t v = v0 + lane;
        const bool empty = v < to && a.start[v] == a.start[v + 1];
        if (empty) {
            G* row = dtable + v * a.ld_table;
            for (uint32_t at = 0; at < bytes; at += kZeroBytes)
                bulk_store(reinterpret_cast<uint8_t*>(row) + at, zeros, min(bytes - at, (uint32_t)kZeroBytes));
            for (int c = (int)(bytes / sizeof(G)); c < a.dim; ++c) from_float(row + c, 0.f);
        }
        bulk_commit();
        bulk_wait_all<4>();
    }
    bulk_wait_all<0>();
}

// `n` sums (n = 4 or 8) of columns [c, c + n) of a token's row to dtable, or onto what is there.
template <int N, class G>
__device__ __forceinline__ void put(const GradArgs& a, G* row, int c, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] *= a.scale;
    if (a.accumulate) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + i < a.dim) f[i] += to_float(row[c + i]);
    }
    if (N == 8 && c + N <= a.dim) {
        float g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = f[i % N];
        Vec8<G>::store(row + c, g);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + i < a.dim) from_float(row + c + i, f[i]);
    }
}

constexpr int kSumWarps = 7;

// A frequent token's segment, by all summing warps of a block: each takes a run of the rows before the first whole piece, of
// the pieces, and of the rows after the last one; the warps' sums are added in order.
template <class T, class G>
__device__ __forceinline__ void sum_frequent(const GradArgs& a, const Used& u, int seg, const T* __restrict__ dout, G* __restrict__ dtable,
                                             float (*part)[Seg<T, false>::kColumns], int warp, int lane) {
    constexpr int K = Seg<T, false>::K, kColumns = Seg<T, false>::kColumns;
    const int c0 = seg * kColumns + lane * 8;
    const int64_t lo = u.lo, hi = u.hi;
    int64_t first = (lo + kPiece - 1) / kPiece, last = hi / kPiece;
    const bool whole = first < last;
    if (!whole) first = last = 0;
    float acc[K][8] = {};
    auto share = [&](int64_t from, int64_t to, int w) { return from + (to - from) * w / kSumWarps; };
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const int64_t from = side == 0 ? lo : whole ? last * kPiece : hi, to = side == 0 && whole ? first * kPiece : hi;
        add_rows<T, false>(acc, a.rows, share(from, to, warp), share(from, to, warp + 1), dout, a.ld, c0, a.dim, lane);
    }
#pragma unroll 4
    for (int64_t p = share(first, last, warp); p < share(first, last, warp + 1); ++p) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (c0 + k * 256 < a.dim) {
                Vec8<float> x;
                x.load(a.pieces + p * a.ldp + c0 + k * 256);
                float f[8];
                x.get(f);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[k][i] += f[i];
            }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) Vec8<float>::store(part[warp] + k * 256 + lane * 8, acc[k]);
    asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
    for (int c = threadIdx.x * 4; c < kColumns; c += kSumWarps * 128) {
        if (seg * kColumns + c >= a.dim) break;
        float f[4] = {};
        for (int w = 0; w < kSumWarps; ++w) {
            const float4 x = *reinterpret_cast<const float4*>(part[w] + c);
            f[0] += x.x, f[1] += x.y, f[2] += x.z, f[3] += x.w;
        }
        put(a, dtable + (int64_t)u.token * a.ld_table, seg * kColumns + c, f);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
}

// The other tokens, a warp for each and segment.  Rows that fit a narrow segment take it, for the rows in flight.
template <class T, class G, bool WIDE>
__device__ __forceinline__ void sum_seldom(const GradArgs& a, int64_t often, const T* __restrict__ dout, G* __restrict__ dtable, int warp,
                                           int lane) {
    constexpr int K = Seg<T, WIDE>::K;
    const int segs = WIDE ? a.wide_segs : 1;
    const int64_t units = (int64_t)a.used[0] * segs, stride = (int64_t)gridDim.x * kSumWarps;
    // blocks with one frequent segment less begin first
    const int64_t turn = (int64_t)((blockIdx.x + gridDim.x - (uint32_t)(often % gridDim.x)) % gridDim.x) * kSumWarps + warp;
    Used next{};
    if (turn < units) next = a.list[turn / segs];
    for (int64_t unit = turn; unit < units; unit += stride) {
        const Used u = next;
        if (unit + stride < units) next = a.list[(unit + stride) / segs];
        const int c0 = (int)(unit % segs) * (K * 256) + lane * 8;
        float acc[K][8] = {};
        add_rows<T, WIDE>(acc, a.rows, u.lo, u.hi, dout, a.ld, c0, a.dim, lane);
#pragma unroll
        for (int k = 0; k < K; ++k) put(a, dtable + (int64_t)u.token * a.ld_table, c0 + k * 256, acc[k]);
    }
}

template <class T, class G>
__global__ void __launch_bounds__(256, 2) embed_rows_kernel(GradArgs a, const T* __restrict__ dout, G* __restrict__ dtable) {
    __shared__ __align__(16) uint8_t zeros[kZeroBytes];
    __shared__ __align__(16) float part[kSumWarps][Seg<T, false>::kColumns];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp == kSumWarps) {
        if (a.accumulate) return;
        const int64_t share = (a.vocab + gridDim.x - 1) / gridDim.x, from = (int64_t)blockIdx.x * share;
        write_zeros(a, zeros, from, min(from + share, (int64_t)a.vocab), dtable, lane);
        return;
    }
    const int64_t often = (int64_t)a.used[1] * a.segs;
    for (int64_t unit = blockIdx.x; unit < often; unit += gridDim.x) {
        const int64_t which = unit / a.segs;
        sum_frequent<T, G>(a, a.list[a.room - 1u - (uint32_t)which], (int)(unit - which * a.segs), dout, dtable, part, warp, lane);
    }
    if (a.segs == 1) sum_seldom<T, G, false>(a, often, dout, dtable, warp, lane);
    else sum_seldom<T, G, true>(a, often, dout, dtable, warp, lane);
}

// ---- host side ------------------------------------------------------------------------------------------------

struct EmbedScratch {
    uint32_t *key_a, *row_a, *key_b, *row_b, *hist, *start, *used;
    Used* list;
    float* pieces;  // [n_rows / kPiece][ldp]
    int64_t ldp;
};

size_t carve_embed(const rapid_embed_desc_t& d, void* base, EmbedScratch* out) {
    size_t off = 0;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* q = p ? p + off : nullptr;
        off = align_up(off + bytes, 256);
        return q;
    };
    EmbedScratch s;
    const size_t n = (size_t)d.n_rows;
    s.key_a = reinterpret_cast<uint32_t*>(take(n * 4));
    s.row_a = reinterpret_cast<uint32_t*>(take(n * 4));
    s.key_b = reinterpret_cast<uint32_t*>(take(n * 4));
    s.row_b = reinterpret_cast<uint32_t*>(take(n * 4));
    s.hist = reinterpret_cast<uint32_t*>(take((size_t)kMaxSortBlocks * kBins * 4));
    s.start = reinterpret_cast<uint32_t*>(take(((size_t)d.vocab + 1) * 4));
    s.used = reinterpret_cast<uint32_t*>(take(8));
    s.list = reinterpret_cast<Used*>(take((n < (size_t)d.vocab ? n : (size_t)d.vocab) * sizeof(Used)));
    s.ldp = (int64_t)align_up((size_t)d.dim, 8);
    s.pieces = reinterpret_cast<float*>(take(n / kPiece * (size_t)s.ldp * 4));
    if (out) *out = s;
    return off;
}

rapid_status_t check_embed(const rapid_embed_desc_t* d, bool bwd) {
    if (!d || d->n_rows <= 0 || d->vocab <= 0 || d->dim <= 0 || d->reserved != 0) return RAPID_ERR_INVALID_ARG;
    if (d->dtype != RAPID_F32 && d->dtype != RAPID_BF16) return RAPID_ERR_INVALID_ARG;
    if (d->flags & ~(uint32_t)(RAPID_EMBED_DTABLE_BF16 | RAPID_EMBED_ACCUMULATE)) return RAPID_ERR_INVALID_ARG;
    if ((d->flags & RAPID_EMBED_DTABLE_BF16) && d->dtype != RAPID_BF16) return RAPID_ERR_INVALID_ARG;
    if (!isfinite(d->scale) || d->ld_table < d->dim || d->ld_rows < d->dim) return RAPID_ERR_INVALID_ARG;
    if (d->n_rows > 0x7fffffffll || d->vocab > (1 << 27) - 2 || d->dim > (1 << 24)) return RAPID_ERR_UNSUPPORTED;
    // far beyond any device's memory; keeps every size below in 64 bits
    if (d->ld_table > (1ll << 56) / d->vocab || d->ld_rows > (1ll << 56) / d->n_rows) return RAPID_ERR_UNSUPPORTED;
    const size_t rows = elem_size(d->dtype);
    const size_t table = !bwd ? rows : (d->flags & RAPID_EMBED_DTABLE_BF16) ? 2 : 4;
    if ((size_t)d->ld_rows * rows % 16 != 0 || (size_t)d->ld_table * table % 16 != 0) return RAPID_ERR_ALIGNMENT;
    return RAPID_OK;
}

// blocks of 8 warps, one unit a warp; false when the grid would not fit
bool blocks_of_8(int64_t units, unsigned* grid) {
    const int64_t b = (units + 7) / 8;
    *grid = (unsigned)b;
    return b <= 0x7fffffffll;
}

template <class T, class G>
rapid_status_t run_bwd(const rapid_embed_desc_t& d, const int32_t* tokens, const uint8_t* mask, const T* dout, G* dtable,
                       const EmbedScratch& w, int sms, cudaStream_t st) {
    const SortShape s = sort_shape(d.n_rows, d.vocab);
    GradArgs g{};
    g.n_rows = d.n_rows;
    g.segs = (d.dim + Seg<T, false>::kColumns - 1) / Seg<T, false>::kColumns;
    g.wide_segs = (d.dim + Seg<T, true>::kColumns - 1) / Seg<T, true>::kColumns;
    g.room = (uint32_t)(d.n_rows < d.vocab ? d.n_rows : d.vocab);
    g.dim = d.dim;
    g.vocab = d.vocab;
    g.ld = d.ld_rows;
    g.ldp = w.ldp;
    g.ld_table = d.ld_table;
    g.scale = d.scale;
    g.accumulate = (d.flags & RAPID_EMBED_ACCUMULATE) != 0;
    g.keys = (s.passes & 1) ? w.key_a : w.key_b;
    g.rows = (s.passes & 1) ? w.row_a : w.row_b;
    g.start = w.start;
    g.used = w.used;
    g.list = w.list;
    g.pieces = w.pieces;
    const int64_t token_blocks = d.vocab / kTokensPerBlock + 1;  // vocab + 1 bounds
    const int64_t prepare = token_blocks + (d.n_rows / kPiece * g.segs + 7) / 8;
    if (prepare > 0x7fffffffll) return RAPID_ERR_UNSUPPORTED;

    SortArgs a{};
    a.tokens = tokens;
    a.mask = mask;
    a.vocab = d.vocab;
    a.hist = w.hist;
    a.used = w.used;
    if (s.blocks == 1) {
        sort_one_block_kernel<<<1, kSortThreads, 0, st>>>(a, s, w.key_a, w.row_a, w.key_b, w.row_b);
    } else {
        for (int p = 0; p < s.passes; ++p) {
            a.shift = p * kRadixBits;
            a.key_in = p == 0 ? nullptr : (p & 1) ? w.key_a : w.key_b;
            a.row_in = p == 0 ? nullptr : (p & 1) ? w.row_a : w.row_b;
            a.key_out = (p & 1) ? w.key_b : w.key_a;
            a.row_out = (p & 1) ? w.row_b : w.row_a;
            sort_hist_kernel<<<s.blocks, kSortThreads, 0, st>>>(a, s);
            sort_scatter_kernel<<<s.blocks, kSortThreads, 0, st>>>(a, s);
        }
    }
    embed_prepare_kernel<T><<<(unsigned)prepare, 256, 0, st>>>(g, (int)token_blocks, dout);
    embed_rows_kernel<T, G><<<2 * sms, 256, 0, st>>>(g, dout, dtable);
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}

}  // namespace
}  // namespace policy
}  // namespace rapid

using namespace rapid;
using namespace rapid::policy;

extern "C" rapid_status_t rapid_embedding_fwd(const rapid_embed_desc_t* desc, const int32_t* tokens, const uint8_t* mask,
                                              const void* table, void* out, rapid_stats_t* stats, void* stream) {
    rapid_status_t s = check_embed(desc, false);
    if (s != RAPID_OK) return s;
    if (!tokens || !table || !out) return RAPID_ERR_INVALID_ARG;
    if (!aligned(table, 16) || !aligned(out, 16) || !aligned(tokens, 4) || !aligned(stats, 8)) return RAPID_ERR_ALIGNMENT;
    const rapid_embed_desc_t& d = *desc;
    const int64_t es = (int64_t)elem_size(d.dtype);
    if (matrices_overlap(table, d.vocab, d.dim * es, d.ld_table * es, out, d.n_rows, d.dim * es, d.ld_rows * es)) return RAPID_ERR_INVALID_ARG;
    const int segs = (d.dim + kFwdSeg - 1) / kFwdSeg;
    unsigned grid = 0;
    if (!blocks_of_8(d.n_rows * segs, &grid)) return RAPID_ERR_UNSUPPORTED;
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (clear_stats(stats, st) != cudaSuccess) return RAPID_ERR_CUDA;
    if (d.dtype == RAPID_BF16)
        embed_fwd_kernel<uint16_t><<<grid, 256, 0, st>>>(d.n_rows, segs, d.vocab, d.dim, d.ld_table, d.ld_rows, d.scale, tokens,
                                                         mask, static_cast<const uint16_t*>(table), static_cast<uint16_t*>(out), stats);
    else
        embed_fwd_kernel<float><<<grid, 256, 0, st>>>(d.n_rows, segs, d.vocab, d.dim, d.ld_table, d.ld_rows, d.scale, tokens, mask,
                                                      static_cast<const float*>(table), static_cast<float*>(out), stats);
    return cudaGetLastError() == cudaSuccess ? RAPID_OK : RAPID_ERR_CUDA;
}

extern "C" rapid_status_t rapid_embedding_bwd_workspace_bytes(const rapid_embed_desc_t* desc, size_t* bytes) {
    if (!bytes) return RAPID_ERR_INVALID_ARG;
    rapid_status_t s = check_embed(desc, true);
    if (s != RAPID_OK) return s;
    *bytes = carve_embed(*desc, nullptr, nullptr);
    return RAPID_OK;
}

extern "C" rapid_status_t rapid_embedding_bwd(const rapid_embed_desc_t* desc, const int32_t* tokens, const uint8_t* mask,
                                              const void* dout, void* dtable, void* workspace, size_t workspace_bytes,
                                              void* stream) {
    rapid_status_t s = check_embed(desc, true);
    if (s != RAPID_OK) return s;
    if (!tokens || !dout || !dtable) return RAPID_ERR_INVALID_ARG;
    if (!aligned(dout, 16) || !aligned(dtable, 16) || !aligned(tokens, 4)) return RAPID_ERR_ALIGNMENT;
    const rapid_embed_desc_t& d = *desc;
    const bool grad_bf16 = (d.flags & RAPID_EMBED_DTABLE_BF16) != 0;
    const int64_t es = (int64_t)elem_size(d.dtype), gs = grad_bf16 ? 2 : 4;
    if (matrices_overlap(dout, d.n_rows, d.dim * es, d.ld_rows * es, dtable, d.vocab, d.dim * gs, d.ld_table * gs)) return RAPID_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return RAPID_ERR_WORKSPACE;
    EmbedScratch w;
    if (workspace_bytes < carve_embed(d, workspace, &w)) return RAPID_ERR_WORKSPACE;
    int sms = 0;
    if ((s = check_device(&sms)) != RAPID_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d.dtype == RAPID_F32)
        return run_bwd(d, tokens, mask, static_cast<const float*>(dout), static_cast<float*>(dtable), w, sms, st);
    if (grad_bf16)
        return run_bwd(d, tokens, mask, static_cast<const uint16_t*>(dout), static_cast<uint16_t*>(dtable), w, sms, st);
    return run_bwd(d, tokens, mask, static_cast<const uint16_t*>(dout), static_cast<float*>(dtable), w, sms, st);
}
