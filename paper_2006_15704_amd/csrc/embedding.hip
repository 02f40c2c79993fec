// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   out[t, :]  = scale * table[id_t, :]                  (zeros for an id outside the table)
//   grad[r, :] = scale * sum of dout[t, :] over the tokens t with id_t = r, t ascending
//
// Both move rows and reuse nothing: they are bound by memory.  What the
// gradient needs besides is the tokens sorted by row, so that every row of
// the gradient is summed in registers and written once, without atomics on
// values: the sum's order is the same in every run.
#include "../../include/ddp_gfx950.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "elem.h"

namespace ddp {
int32_t fail_without_context(int32_t code, const std::string& msg);   // ddp_api.hip
}

namespace {

using namespace ddp;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int64_t kMaxRows = int64_t(1) << 23, kMaxTokens = int64_t(1) << 22, kMaxWidth = int64_t(1) << 20;

template <typename Id>
__device__ __forceinline__ int64_t row_of(const Id* ids, int64_t t) { return static_cast<int64_t>(*(DDP_GLOBAL_MEM const Id*)(ids + t)); }

// The columns of a wave: GROUPS vectors of N elements a lane, 64 N columns apart.  The vector that would reach over the end of a row
// is moved back to end with it, so that every access is a whole vector; what it shares with the vector in front is
// read twice and written once (`own`: elements from here on are the lane's to write).  Rows of fewer than N columns take N = 1.
template <int N, int GROUPS>
struct Columns {
    int at[GROUPS];
    int own[GROUPS];                             // N: nothing here
    __device__ __forceinline__ Columns(int first, int width) {
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            const int c = first + (s * 64 + static_cast<int>(threadIdx.x & 63)) * N;
            at[s] = c + N <= width ? c : width - N;
            own[s] = c >= width ? N : c - at[s];
        }
    }
};

template <int DT, bool NT, int N>
__device__ __forceinline__ void store_own(char* row, int at, int own, const float (&x)[N]) {
    char* to = row + at * ElemBytes<DT>::value;
    if (own == 0) {
        store_some<DT, N, NT>(to, N, x);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= own) store_one<DT>(to + i * ElemBytes<DT>::value, x[i]);
    }
}
// N = 1 of a 16-bit type is half a dword: no vector access.
template <int DT, int N> struct Vector {
    Parts<DT, N> raw;
    template <bool NT = false>
    __device__ __forceinline__ void load(const char* p) { raw = load_parts<DT, N, NT>(p); }
    __device__ __forceinline__ void get(float (&x)[N]) const { widen<DT, N>(raw, x); }
};
template <int DT> struct Vector<DT, 1> {
    float x1;
    template <bool NT = false>
    __device__ __forceinline__ void load(const char* p) { x1 = load_one<DT>(p); }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = x1; }
};
template <int DT, bool NT>
__device__ __forceinline__ void store_own(char* row, int at, int own, const float (&x)[1]) {
    if (own == 0) store_one<DT>(row + at * ElemBytes<DT>::value, x[0]);
}

// ---- lookup ----

// Rows that the caches cannot keep for the next kernel are stored with the non-temporal hint: 16384 rows of 1024, binary32 table,
// bfloat16 rows (33 MB) 11.2 us with it, 13.2 without.
constexpr int64_t kStreamBytes = int64_t(4) << 20;

// A wave takes a row; all its loads (up to 1024 columns) are on the way together.  Those 16384 rows are 54 MB, 4.9 TB/s: what is left is
// the latency of an id and then its row, once a wave.  One row alone 1.9 us.
template <typename Id, int WT, int OT, int N>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const Id* ids, int64_t tokens, const char* table, int64_t rows, int width,
                                                          int64_t table_stride, float scale, char* out, int64_t out_stride, int stream) {
    constexpr int GROUPS = N == 1 ? 1 : 16 / N;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (t >= tokens) return;
    const int64_t r = row_of(ids, t);
    const bool named = r >= 0 && r < rows;
    const char* from = table + (named ? r : 0) * table_stride * ElemBytes<WT>::value;
    char* to = out + t * out_stride * ElemBytes<OT>::value;
    for (int c = 0; c < width; c += 64 * N * GROUPS) {
        const Columns<N, GROUPS> at(c, width);
        Vector<WT, N> v[GROUPS];
#pragma unroll
        for (int s = 0; s < GROUPS; ++s)
            if (at.own[s] < N) v[s].load(from + at.at[s] * ElemBytes<WT>::value);
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            if (at.own[s] == N) continue;
            float x[N];
            v[s].get(x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = named ? x[i] * scale : 0.0f;
            if (stream) store_own<OT, true>(to, at.at[s], at.own[s], x);
            else store_own<OT, false>(to, at.at[s], at.own[s], x);
        }
    }
}

// Rows of up to half a wave's vectors: a thread takes one vector of one token.  (100 thousand rows of 64 in bfloat16: 5 us, with a wave
// a row 18.)
template <typename Id, int WT, int OT, int N>
__global__ __launch_bounds__(kThreads) void narrow_lookup_kernel(const Id* ids, unsigned tokens, const char* table, int64_t rows, int width, int64_t table_stride,
                                                                 float scale, char* out, int64_t out_stride, int stream) {
    const unsigned vectors = (width + N - 1) / N, i = blockIdx.x * kThreads + threadIdx.x, t = i / vectors;
    if (t >= tokens) return;
    const int c = static_cast<int>(i - t * vectors) * N, at = min(c, width - N);
    const int64_t r = row_of(ids, t);
    const bool named = r >= 0 && r < rows;
    Vector<WT, N> v;
    v.load(table + ((named ? r : 0) * table_stride + at) * ElemBytes<WT>::value);
    float x[N];
    v.get(x);
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = named ? x[k] * scale : 0.0f;
    char* to = out + t * out_stride * ElemBytes<OT>::value;
    if (stream) store_own<OT, true>(to, at, c - at, x);
    else store_own<OT, false>(to, at, c - at, x);
}

// ---- sums of tokens' rows ----

struct SumArgs {
    const uint32_t* first;
    const uint32_t* sorted;
    const void* ids;
    const char* dout;
    char* grad;
    const uint32_t* split;
    float* partial;                              // [windows][2][width], of the parts that `split` lists
    int64_t tokens, rows, dout_stride, grad_stride, padding;
    int32_t width, windows, window_blocks, row_blocks, rows_per_block, add;
    int32_t units, window_units, log2_blocks, log2_run; // units: column ranges of a wave in a row
    int32_t shift, bucket_bits, log2_window;     // of the sort
    float scale;
};

// U: tokens whose rows are on the way together.
template <int FT, int N, int GROUPS, int U = 8>
struct Sum {
    float acc[GROUPS][N] = {};

    __device__ __forceinline__ void load(Vector<FT, N> (&v)[GROUPS], const SumArgs& a, const Columns<N, GROUPS>& at, uint32_t token) {
        const char* row = a.dout + static_cast<int64_t>(token) * a.dout_stride * ElemBytes<FT>::value;
#pragma unroll
        for (int s = 0; s < GROUPS; ++s)
            if (at.own[s] < N) v[s].load(row + at.at[s] * ElemBytes<FT>::value);
    }
    __device__ __forceinline__ void add(const Vector<FT, N> (&v)[GROUPS], const Columns<N, GROUPS>& at) {
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            if (at.own[s] == N) continue;
            float x[N];
            v[s].get(x);
#pragma unroll
            for (int k = 0; k < N; ++k) acc[s][k] += x[k];
        }
    }
    // The tokens that `token(i)` gives for i = 0 .. n-1, in this order; n and token(i) are the same in all lanes.
    template <typename Token>
    __device__ __forceinline__ void tokens(const SumArgs& a, const Columns<N, GROUPS>& at, int n, Token token) {
        for (int i = 0; i < n; i += U) {
            Vector<FT, N> v[U][GROUPS];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u < n) load(v[u], a, at, token(i + u));
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u < n) add(v[u], at);
        }
    }
    template <int GT>
    __device__ __forceinline__ void put(const SumArgs& a, const Columns<N, GROUPS>& at, int64_t row) {
        char* to = a.grad + row * a.grad_stride * ElemBytes<GT>::value;
        if (a.add) {
            Vector<GT, N> old[GROUPS];
#pragma unroll
            for (int s = 0; s < GROUPS; ++s)
                if (at.own[s] < N) old[s].load(to + at.at[s] * ElemBytes<GT>::value);
#pragma unroll
            for (int s = 0; s < GROUPS; ++s) {
                if (at.own[s] == N) continue;
                float x[N];
                old[s].get(x);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[s][k] = acc[s][k] * a.scale + x[k];
                store_own<GT, true>(to, at.at[s], at.own[s], acc[s]);
            }
            return;
        }
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            if (at.own[s] == N) continue;
#pragma unroll
            for (int k = 0; k < N; ++k) acc[s][k] *= a.scale;
            store_own<GT, true>(to, at.at[s], at.own[s], acc[s]);
        }
    }
};

// Where a row comes in the sort, and the row there.
__device__ __forceinline__ int64_t place_of(const SumArgs& a, int64_t row) { return (row & ((int64_t(1) << a.bucket_bits) - 1)) << a.shift | row >> a.bucket_bits; }
__device__ __forceinline__ int64_t row_at(const SumArgs& a, int64_t place) { return (place & ((int64_t(1) << a.shift) - 1)) << a.bucket_bits | place >> a.shift; }

__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0));
}
__device__ __forceinline__ uint32_t wave_inclusive_sum(uint32_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) {
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), lane));
}

// Vector i of a block's rows one after the other: zeros at its place in the gradient.  row_of_block(j) is the block's row j, or -1
// where that is not to be zeroed.
template <int GT, int N, typename Row>
__device__ __forceinline__ void zero_vector(const SumArgs& a, unsigned i, Row row_of_block) {
    const unsigned vectors = (a.width + N - 1) / N, j = i / vectors;
    const int64_t row = row_of_block(static_cast<int>(j));
    if (row < 0) return;
    const int at = min(static_cast<int>(i - j * vectors) * N, a.width - N);     // (the last two may overlap: zeros both)
    const float zeros[N] = {};
    store_own<GT, true>(a.grad + row * a.grad_stride * ElemBytes<GT>::value, at, 0, zeros);
}

// ---- few tokens: every block looks through all of them ----
//
// Rows go round 2^log2_blocks blocks in runs of 2^log2_run (rows of frequent tokens are neighbours in many vocabularies: they
// go to different blocks).  A block lists the tokens of its rows, t ascending, and its waves sum a row each; rows of many tokens
// are split over the block's waves and joined in LDS, in order.  4096 tokens into 30522 rows of 1024 (133 MB, nearly all of it zeros
// that are written): 30 us, 4.5 TB/s; with one token 23.1, 5.4 TB/s (rows one by one instead of in pairs 24.3, by 30 instead of 60 a block 26.9).

constexpr int kScanThreads = 512, kScanWaves = kScanThreads / 64;
constexpr int kScanTokens = 4096;
constexpr int kScanEach = kScanTokens / kScanThreads;
constexpr int64_t kScanBlockBytes = 8192;        // to move by each of them
constexpr int kScanBlocks = 4096;                // blocks to have where there are column ranges to go round
constexpr int kScanAlone = 16;                   // tokens of a row that one wave sums
constexpr int kScanRows = 32;                    // rows of 1024 columns that a block has at most, single (up to 1024 of fewer columns); twice that in pairs

template <typename Id, int FT, int GT, int N>
__global__ __launch_bounds__(kScanThreads, 6) void scan_sum_kernel(SumArgs a) {
    __shared__ uint32_t list[kScanTokens];           // row in the block << 16 | token
    __shared__ uint32_t wave_count[kScanWaves];
    __shared__ float part[kScanWaves][64 * N];
    extern __shared__ uint32_t counts[];             // of the tokens of each row
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.x;
    const int run = (1 << a.log2_run) - 1;
    const int nrows = static_cast<int>(((a.rows - 1) >> (a.log2_blocks + a.log2_run)) + 1) << a.log2_run;
    auto block_of = [&](int64_t row) { return row >> a.log2_run & ((int64_t(1) << a.log2_blocks) - 1); };
    auto index_of = [&](int row) { return row >> (a.log2_run + a.log2_blocks) << a.log2_run | (row & run); };
    auto row_of_block = [&](int j) { return ((static_cast<int64_t>(j >> a.log2_run) << a.log2_blocks | b) << a.log2_run) + (j & run); };
    const int per_wave = static_cast<int>((a.tokens + kScanThreads - 1) / kScanThreads) * 64;
    for (int i = threadIdx.x; i < nrows; i += kScanThreads) counts[i] = 0;
    int64_t id[kScanEach];
    int row[kScanEach];
#pragma unroll
    for (int k = 0; k < kScanEach; ++k) {
        const int t = wave * per_wave + k * 64 + lane;
        id[k] = k * 64 < per_wave && t < a.tokens ? row_of(static_cast<const Id*>(a.ids), t) : -1;
    }
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < kScanEach; ++k) {
        row[k] = id[k] < 0 || id[k] >= a.rows || id[k] == a.padding || block_of(id[k]) != b ? -1 : static_cast<int>(id[k]);
        mine += __popcll(__ballot(row[k] >= 0));
    }
    if (lane == 0) wave_count[wave] = mine;
    __syncthreads();
    uint32_t next = 0, listed = 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) {
        if (w < wave) next += wave_count[w];
        listed += wave_count[w];
    }
#pragma unroll
    for (int k = 0; k < kScanEach; ++k) {
        const uint64_t hits = __ballot(row[k] >= 0);
        if (row[k] >= 0) {
            list[next + lanes_below(hits)] = static_cast<uint32_t>(index_of(row[k])) << 16 | static_cast<uint32_t>(wave * per_wave + k * 64 + lane);
            atomicAdd(&counts[index_of(row[k])], 1u);
        }
        next += __popcll(hits);
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(static_cast<int>(listed));
    // the column ranges of the block: blockIdx.y, + gridDim.y, ...
    const int units = (a.units - static_cast<int>(blockIdx.y) + static_cast<int>(gridDim.y) - 1) / static_cast<int>(gridDim.y);
    auto first_column = [&](int i) { return (static_cast<int>(blockIdx.y) + i * static_cast<int>(gridDim.y)) * (64 * N); };
    // rows of no tokens: the blocks of one set of rows and other columns share them
    if (!a.add) {
        const unsigned vectors = nrows * ((a.width + N - 1) / N), step = kScanThreads * gridDim.y;
        for (unsigned i = blockIdx.y * kScanThreads + threadIdx.x; i < vectors; i += step)
            zero_vector<GT, N>(a, i, [&](int j) { return counts[j] == 0 && row_of_block(j) < a.rows ? row_of_block(j) : -1; });
    }
    if (n == 0) return;
    // rows of few tokens, a wave for each and each range
    int turn = 0;
    for (int j0 = 0; j0 < nrows; j0 += 64) {
        const uint32_t here = counts[min(j0 + lane, nrows - 1)];
        for (uint64_t some = __ballot(j0 + lane < nrows && here > 0 && here <= kScanAlone); some != 0; some &= some - 1) {
            const int l = __ffsll(static_cast<unsigned long long>(some)) - 1, j = j0 + l;
            for (int unit = 0; unit < units; ++unit, ++turn) {
                if (turn % kScanWaves != wave) continue;
                int left = static_cast<int>(lane_value(here, l));
                const Columns<N, 1> at(first_column(unit), a.width);
                Sum<FT, N, 1> sum;
                for (int i = 0; left > 0; i += 64) {
                    const uint32_t e = list[min(i + lane, n - 1)];
                    uint64_t hits = __ballot(i + lane < n && e >> 16 == static_cast<uint32_t>(j));
                    const int found = __popcll(hits);
                    left -= found;
                    sum.tokens(a, at, found, [&](int) {
                        const int k = __ffsll(static_cast<unsigned long long>(hits)) - 1;
                        hits &= hits - 1;
                        return lane_value(e, k) & 0xFFFFu;
                    });
                }
                sum.template put<GT>(a, at, row_of_block(j));
            }
        }
    }
    if (n <= kScanAlone) return;
    for (int j0 = 0; j0 < nrows; j0 += 64) {
        uint64_t crowded = __ballot(j0 + lane < nrows && counts[min(j0 + lane, nrows - 1)] > kScanAlone);
        for (; crowded != 0; crowded &= crowded - 1) {
            const int j = j0 + __ffsll(static_cast<unsigned long long>(crowded)) - 1;
            const int count = __builtin_amdgcn_readfirstlane(static_cast<int>(counts[j]));
            const int share = (count + kScanWaves - 1) / kScanWaves, from = wave * share, to = min(from + share, count);
            for (int unit = 0; unit < units; ++unit) {
                const Columns<N, 1> at(first_column(unit), a.width);
                Sum<FT, N, 1> sum;
                int seen = 0;                        // the row's tokens so far
                for (int i = 0; i < n && seen < to; i += 64) {
                    const uint32_t e = list[min(i + lane, n - 1)];
                    const bool hit = i + lane < n && e >> 16 == static_cast<uint32_t>(j);
                    const uint64_t all = __ballot(hit);
                    const int order = seen + lanes_below(all);
                    uint64_t hits = __ballot(hit && order >= from && order < to);
                    seen += __popcll(all);
                    sum.tokens(a, at, __popcll(hits), [&](int) {
                        const int l = __ffsll(static_cast<unsigned long long>(hits)) - 1;
                        hits &= hits - 1;
                        return lane_value(e, l) & 0xFFFFu;
                    });
                }
                if (wave > 0) {
#pragma unroll
                    for (int k = 0; k < N; ++k) part[wave][k * 64 + lane] = sum.acc[0][k];
                }
                __syncthreads();
                if (wave == 0) {
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        for (int w = 1; w < kScanWaves; ++w) sum.acc[0][k] += part[w][k * 64 + lane];
                    sum.template put<GT>(a, at, row_of_block(j));
                }
                __syncthreads();
            }
        }
    }
}

// ---- more tokens: sorted by row ----
//
// Rows are put into 2^bucket_bits buckets by their low bits, so that the frequent rows, which are neighbours in many
// vocabularies, come into different ones; the order in which `sorted` and `first` have the rows is by bucket, then by what is left
// of the row (`place_of`, `row_at`).  A block sorts a chunk of tokens by bucket; starts[chunk][b] is where
// bucket b starts in the chunk's part of `list`, which is also the number of the chunk's tokens in the buckets before it: summed
// over the chunks it is where the bucket starts among all tokens, so no scan over buckets is needed.  A block then
// gathers a bucket's tokens chunk by chunk (t ascending) and sorts them by row.

// A row of up to 2^log2_window tokens is summed by one wave (and column range).  Rows of more are split at multiples of the window in the
// sorted tokens, their parts go through `partial` and are joined by another launch.  split[w][0] is 1 + the place of the row
// that reaches back before window w, split[w][1] of the one that starts in it, 0 where there is no such row of more than a window's
// tokens (two of them cannot start in one window).  Windows are short, so that a wave's rounds of loads are few, but where all rows
// have many tokens the parts of a row would be.
constexpr int kLog2Window = 5, kLog2LongWindow = 7;
// 65536 tokens into two rows of 1024, us, windows of 32 / 128: sums 52 / 48, joins 32 / 10; but 42858 into five of 26 have too few
// windows for the chip: 28 / 40 in all.  Over 192 calls (8192 to 131072 tokens, rows of 512 to 8192 bytes, 48 tokens a row and more): with
// fewer than 600 column ranges of windows 32 wins, by up to half (8192 into 27 of 512 in bfloat16 21.5 / 30.8); at 1024 the two are within a tenth
// (65536 into 128 of 1024 42.8 / 40.5), from 2048 on 128 wins by a tenth to a fifth (131072 into 256 of 1024 68 / 60), and one row takes half
// the time (65536 into one of 1024 82 / 49).  Where the rule is not the better one it loses up to a quarter (48 to 255 tokens a row, many
// ranges: 65536 into 682 of 4096 147 / 119; rows of 512 bytes: 131072 into 436 32 / 38), for one row of few ranges a half (71 / 47).
inline int log2_window(int64_t tokens, int64_t rows, int64_t ranges) {
    return tokens / rows >= 256 && (tokens >> kLog2LongWindow) * ranges >= 1024 ? kLog2LongWindow : kLog2Window;
}

constexpr int kChunk = 1024;
constexpr int kMaxBuckets = 8192;                // 32 KiB of counters
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kSortRows = 1024;                  // places of a bucket, at most
constexpr int kSortCache = 4096;                 // tokens of a bucket held in LDS
constexpr int kTokenBits = 22;
constexpr uint32_t kTokenMask = (1u << kTokenBits) - 1;
static_assert(kMaxTokens <= int64_t(1) << kTokenBits && kSortRows <= 1 << (32 - kTokenBits), "an entry is 32 bits");

struct SortArgs {
    const void* ids;
    int64_t tokens, rows, padding;
    int32_t shift, buckets, bucket_bits, chunks; // buckets of 2^shift places
    int32_t log2_window;
    uint16_t* starts;                            // [chunks][buckets + 1]
    uint32_t* list;                              // [tokens] by chunk, by bucket: entries, place in the bucket << 22 | token
    uint32_t* gathered;                          // [tokens] by bucket, t ascending (buckets that LDS does not hold)
    uint32_t* sorted;                            // [tokens] by place, t ascending
    uint32_t* first;                             // [places + 1] where each place's row starts in `sorted`
    uint32_t* split;                             // [windows][2] see Split
};

// Lanes of the wave (of those in `active`) that hold the same value of `bits` bits.
__device__ __forceinline__ uint64_t peers(uint32_t value, int bits, uint64_t active) {
    uint64_t same = active;
    for (int b = 0; b < bits; ++b) {
        const bool set = value >> b & 1u;
        const uint64_t ones = __ballot(set);
        same &= set ? ones : ~ones;
    }
    return same;
}

template <typename Id>
__global__ __launch_bounds__(kChunk) void chunk_sort_kernel(SortArgs a) {
    extern __shared__ uint32_t count[];              // [buckets]
    __shared__ uint32_t wave_sum[kChunk / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kChunk + tid;
    const int64_t row = t < a.tokens ? row_of(static_cast<const Id*>(a.ids), t) : -1;
    const bool in = row >= 0 && row < a.rows && row != a.padding;
    for (int i = tid; i < a.buckets; i += kChunk) count[i] = 0;
    const int splits = 2 * kChunk >> a.log2_window;
    if (tid < splits) a.split[static_cast<int64_t>(blockIdx.x) * splits + tid] = 0;
    const uint32_t b = in ? static_cast<uint32_t>(row) & (a.buckets - 1) : 0u;
    const uint64_t same = peers(b, a.bucket_bits, __ballot(in));
    const uint32_t rank = lanes_below(same);
    uint32_t before = 0;
    __syncthreads();
    for (int w = 0; w < kChunk / 64; ++w) {          // the waves in turn: t ascending
        if (w == wave && in) {
            before = count[b];
            if (rank == 0) count[b] = before + __popcll(same);
        }
        __syncthreads();
    }
    // exclusive scan: a thread sums a run of buckets
    const int run = (a.buckets + kChunk - 1) / kChunk;
    const int from = min(tid * run, a.buckets), to = min(from + run, a.buckets);
    uint32_t sum = 0;
    for (int i = from; i < to; ++i) sum += count[i];
    const uint32_t upto = wave_inclusive_sum(sum);
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    uint32_t next = upto - sum;
    for (int w = 0; w < wave; ++w) next += wave_sum[w];
    uint16_t* starts = a.starts + static_cast<int64_t>(blockIdx.x) * (a.buckets + 1);
    for (int i = from; i < to; ++i) {
        const uint32_t n = count[i];
        count[i] = next;
        starts[i] = static_cast<uint16_t>(next);
        next += n;
    }
    if (tid == kChunk - 1) starts[a.buckets] = static_cast<uint16_t>(next);
    __syncthreads();
    if (in) a.list[static_cast<int64_t>(blockIdx.x) * kChunk + count[b] + before + rank] = static_cast<uint32_t>(row) >> a.bucket_bits << kTokenBits | static_cast<uint32_t>(t);
}

// LDS accesses of a wave stay in order; the fence keeps the compiler to it.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return __builtin_amdgcn_readfirstlane(x);
}

// A bucket's counters in LDS: where the next token of each row goes, and where a row of more than a window's tokens starts in `sorted`
// (others: the largest number).
struct RowCounters {
    uint32_t *next, *crowded_from;
};
// Row r of a bucket has n tokens, the first of them at `from` in `sorted`.
__device__ __forceinline__ void row_starts(const SortArgs& a, const RowCounters& rows, int64_t place0, int r, uint32_t from, uint32_t n) {
    a.first[place0 + r] = from;
    const bool crowded = n > 1u << a.log2_window;
    rows.crowded_from[r] = crowded ? from : ~0u;
    if (crowded) a.split[(from >> a.log2_window) * 2 + 1] = 1 + static_cast<uint32_t>(place0 + r);
}
// 64 tokens of a bucket (entries; lanes that are not `in` have none) go to their places behind `base`.
__device__ __forceinline__ void place_tokens(const SortArgs& a, uint32_t* next, const uint32_t* crowded_from, int64_t place0, uint32_t base, uint32_t e, bool in) {
    const uint32_t r = e >> kTokenBits;
    const uint64_t same = peers(r, a.shift, __ballot(in));
    const uint32_t rank = lanes_below(same);
    uint32_t p = 0;
    if (in) p = next[r];
    wave_fence();
    if (in) {
        const uint32_t at = base + p + rank;
        a.sorted[at] = e & kTokenMask;
        if ((at & ((1u << a.log2_window) - 1)) == 0 && crowded_from[r] < at) a.split[(at >> a.log2_window) * 2] = 1 + static_cast<uint32_t>(place0) + r;
        if (rank == 0) next[r] = p + __popcll(same);
    }
    wave_fence();
}

// Up to this many tokens of a bucket are sorted by the block's first wave alone, without barriers (20011 tokens in 1024 buckets:
// 7.7 us, all by whole blocks 10.5; with half this limit the same).
constexpr int kWaveTokens = 256;

// Several blocks (gridDim.y) share the copying where a bucket is one row.
__global__ __launch_bounds__(kSortThreads) void bucket_sort_kernel(SortArgs a) {
    __shared__ uint32_t cache[kSortCache];
    static_assert(kWaveTokens <= kSortCache && kWaveTokens >= 1 << kLog2LongWindow, "a bucket for the block has more tokens than a window");
    __shared__ uint32_t wave_part[kSortWaves], wave_before[kSortWaves];
    __shared__ uint32_t more[kSortThreads], more_from[kSortThreads], more_to[kSortThreads];
    extern __shared__ uint32_t counters[];           // [kSortWaves + 1][rows of a bucket]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nrows = 1 << a.shift;
    const RowCounters rows{counters + wave * nrows, counters + kSortWaves * nrows};
    auto starts_of = [&](int c, int b) { return a.starts + static_cast<int64_t>(c) * (a.buckets + 1) + b; };
    const int b = blockIdx.x;
    const int64_t place0 = static_cast<int64_t>(b) << a.shift;
    uint32_t before = 0, mine = 0;
    for (int c = tid; c < a.chunks; c += kSortThreads) {
        const uint16_t* p = starts_of(c, b);
        before += p[0];
        mine += p[1] - p[0];
    }
    before = wave_sum(before);
    mine = wave_sum(mine);
    if (lane == 0) {
        wave_before[wave] = before;
        wave_part[wave] = mine;
    }
    for (int i = tid; i < kSortWaves * nrows; i += kSortThreads) counters[i] = 0;
    __syncthreads();
    uint32_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        base += wave_before[w];
        total += wave_part[w];
    }
    if (b == a.buckets - 1 && tid == 0) a.first[place0 + nrows] = base + total;
    if (total <= kWaveTokens) {
        if (wave > 0 || blockIdx.y > 0) return;
        uint32_t* tokens = cache;
        uint32_t done = 0;
        for (int c0 = 0; c0 < a.chunks && done < total; c0 += 64) {
            const int c = c0 + lane;
            uint32_t s = 0, n = 0;
            if (c < a.chunks) {
                const uint16_t* p = starts_of(c, b);
                s = p[0];
                n = p[1] - s;
            }
            const uint32_t upto = wave_inclusive_sum(n), to = done + upto - n;
            const uint32_t* from = a.list + static_cast<int64_t>(c) * kChunk + s;
            for (uint32_t i = 0; i < n; i += 4) {
                uint32_t few[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) few[k] = i + k < n ? from[i + k] : 0u;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    if (i + k < n) tokens[to + i + k] = few[k];
            }
            done += lane_value(upto, 63);
        }
        wave_fence();
        for (uint32_t i = lane; i < total; i += 64) atomicAdd(&rows.next[tokens[i] >> kTokenBits], 1u);
        wave_fence();
        uint32_t above = 0;
        for (int r0 = 0; r0 < nrows; r0 += 64) {
            const int r = r0 + lane;
            const uint32_t n = r < nrows ? rows.next[r] : 0u;
            const uint32_t upto = wave_inclusive_sum(n);
            if (r < nrows) {
                row_starts(a, rows, place0, r, base + above + upto - n, n);
                rows.next[r] = above + upto - n;
            }
            above += lane_value(upto, 63);
        }
        wave_fence();
        for (uint32_t i0 = 0; i0 < total; i0 += 64) {
            const bool in = i0 + lane < total;
            place_tokens(a, rows.next, rows.crowded_from, place0, base, in ? tokens[i0 + lane] : 0u, in);
        }
        return;
    }
    // the bucket's tokens in order: a thread copies up to four of its chunk's, the waves together what there is above that
    uint32_t* tokens = a.shift == 0 ? a.sorted + base : total <= kSortCache ? cache : a.gathered + base;     // (a bucket of one row is sorted by then)
    uint32_t done = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += kSortThreads) {
        const int c = c0 + tid;
        uint32_t s = 0, n = 0;
        if (c < a.chunks) {
            const uint16_t* p = starts_of(c, b);
            s = p[0];
            n = p[1] - s;
        }
        const uint32_t upto = wave_inclusive_sum(n);
        __syncthreads();                             // wave_part and `more` are read by then
        if (lane == 63) wave_part[wave] = upto;
        __syncthreads();
        uint32_t to = done + upto - n;
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) to += wave_part[w];
            done += wave_part[w];
        }
        const uint32_t* from = a.list + static_cast<int64_t>(c) * kChunk + s;
        if (static_cast<unsigned>(c) / kSortWaves % gridDim.y != blockIdx.y) n = 0;       // another block's chunk
        uint32_t few[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) few[i] = i < static_cast<int>(n) ? from[i] : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < static_cast<int>(n)) tokens[to + i] = few[i];
        more[tid] = n > 4 ? n - 4 : 0;
        more_from[tid] = s + 4;
        more_to[tid] = to + 4;
        const int rounds = min(kSortThreads, a.chunks - c0);
        if (!__syncthreads_or(n > 4)) continue;
        for (int k = wave; k < rounds; k += kSortWaves) {
            const uint32_t nk = __builtin_amdgcn_readfirstlane(more[k]);
            if (nk == 0) continue;
            const uint32_t* p = a.list + static_cast<int64_t>(c0 + k) * kChunk + more_from[k];
            uint32_t* q = tokens + more_to[k];
            for (uint32_t i0 = 0; i0 < nk; i0 += 256) {
                uint32_t e[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) e[u] = i0 + u * 64 + lane < nk ? p[i0 + u * 64 + lane] : 0u;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i0 + u * 64 + lane < nk) q[i0 + u * 64 + lane] = e[u];
            }
        }
    }
    if (a.shift == 0) {
        if (blockIdx.y > 0) return;
        if (tid == 0) row_starts(a, rows, place0, 0, base, total);
        for (uint32_t w = (base >> a.log2_window) + 1 + tid; w <= (base + total - 1) >> a.log2_window; w += kSortThreads) a.split[w * 2] = 1 + static_cast<uint32_t>(place0);
        return;
    }
    __threadfence_block();
    __syncthreads();
    // counting sort by row: every wave has a stretch of the tokens
    const uint32_t stretch = (total + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
    const uint32_t from = min(wave * stretch, total), to = min(from + stretch, total);
    for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&rows.next[tokens[i] >> kTokenBits], 1u);
    __syncthreads();
    // row by row, within a row wave by wave; the rows' sums are scanned in rounds of one row a thread
    uint32_t above = 0;
    for (int r0 = 0; r0 < nrows; r0 += kSortThreads) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < nrows)
            for (int w = 0; w < kSortWaves; ++w) n += counters[w * nrows + r];
        const uint32_t upto = wave_inclusive_sum(n);
        if (lane == 63) wave_part[wave] = upto;
        __syncthreads();
        uint32_t next = above + upto - n;
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) next += wave_part[w];
            above += wave_part[w];
        }
        __syncthreads();
        if (r < nrows) {
            row_starts(a, rows, place0, r, base + next, n);
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t k = counters[w * nrows + r];
                counters[w * nrows + r] = next;
                next += k;
            }
        }
    }
    __syncthreads();
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const bool in = i0 + lane < to;
        place_tokens(a, rows.next, rows.crowded_from, place0, base, in ? tokens[i0 + lane] : 0u, in);
    }
}

// What the sort leaves is the sums: rows of dout are read once, a row of the gradient is written once.  65536 tokens (59 thousand
// kept) into 30522 rows of 1024, bfloat16: chunks 5.4 us, buckets 12.8, sums 38.8 (183 MB, 4.7 TB/s: the rows are read
// as the tokens lie, and the crowded rows' windows end last), joins 6.3.

constexpr int kRowColumns = 8192;                // of the rows of a block: 8 rows of 1024, at most 64 of fewer, ...
constexpr int kRowBlocks = 1024;                 // ... where that leaves so many blocks

template <int FT, int N>
__device__ __forceinline__ void sum_window(const SumArgs& a, int64_t w, int unit) {
    const uint32_t split[2] = {a.split[w * 2], a.split[w * 2 + 1]};
    const uint32_t w0 = static_cast<uint32_t>(w) << a.log2_window;
    const Columns<N, 1> at(unit * (64 * N), a.width);
    for (int side = 0; side < 2; ++side) {
        if (split[side] == 0) continue;
        const uint32_t from = __builtin_amdgcn_readfirstlane(max(a.first[split[side] - 1], w0));
        const uint32_t to = __builtin_amdgcn_readfirstlane(min(a.first[split[side]], w0 + (1u << a.log2_window)));
        Sum<FT, N, 1> sum;
        for (uint32_t i = from; i < to; i += 64) {
            const uint32_t mine = a.sorted[min(i + (threadIdx.x & 63), to - 1)];
            sum.tokens(a, at, static_cast<int>(min(to - i, 64u)), [&](int k) { return lane_value(mine, k); });
        }
        char* to_part = reinterpret_cast<char*>(a.partial + (w * 2 + side) * static_cast<int64_t>(a.width));
        if (at.own[0] < N) store_own<DDP_FP32, false>(to_part, at.at[0], at.own[0], sum.acc[0]);
    }
}

// The first blocks take windows, the others rows_per_block rows each, row_blocks apart (the frequent rows are neighbours in many
// vocabularies: every block has some of each): a row's sum, or zeros.  Work is a wave's: one row, 64 N columns, 16-byte stores; units this small in
// registers for 8 waves a SIMD did better than wider ones, which end unevenly.
template <int FT, int GT, int N, int WN>
__global__ __launch_bounds__(kThreads) void row_sum_kernel(SumArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (static_cast<int>(blockIdx.x) < a.window_blocks) {
        const int64_t g = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
        if (g / a.window_units < a.windows) sum_window<FT, WN>(a, g / a.window_units, static_cast<int>(g % a.window_units));
        return;
    }
    // lane k knows row k of the block: where its tokens are, and the first of them
    const int64_t block = static_cast<int>(blockIdx.x) - a.window_blocks;
    auto row_of_block = [&](int j) { return block + static_cast<int64_t>(j) * a.row_blocks; };
    const int64_t mine = row_of_block(lane);
    const bool have = lane < a.rows_per_block && mine < a.rows;
    const int64_t place = place_of(a, have ? mine : 0);
    const uint32_t from = a.first[place], count = have ? a.first[place + 1] - from : ~0u;
    const uint32_t token = have && count > 0 ? a.sorted[from] : 0u;
    if (!a.add && __ballot(count == 0) != 0) {
        const unsigned vectors = a.rows_per_block * ((a.width + N - 1) / N);
        for (unsigned i0 = 0; i0 < vectors; i0 += kThreads)                  // all lanes: the counts are in registers
            zero_vector<GT, N>(a, min(i0 + threadIdx.x, vectors - 1), [&](int j) { return __shfl(count, j) == 0u ? row_of_block(j) : -1; });
    }
    int turn = 0;
    for (uint64_t some = __ballot(count - 1u < 1u << a.log2_window); some != 0; some &= some - 1) {
        const int j = __ffsll(static_cast<unsigned long long>(some)) - 1, n = static_cast<int>(lane_value(count, j));
        bool fetched = n == 1;
        uint32_t own = lane_value(token, j);
        for (int unit = 0; unit < a.units; ++unit, ++turn) {
            if (turn % kWaves != wave) continue;
            if (!fetched) own = a.sorted[lane_value(from, j) + min(lane, n - 1)];
            fetched = n <= 64;
            const Columns<N, 1> at(unit * (64 * N), a.width);
            Sum<FT, N, 1> sum;
            sum.tokens(a, at, min(n, 64), [&](int k) { return lane_value(own, k); });
            for (int i = 64; i < n; i += 64) {
                const uint32_t more = a.sorted[lane_value(from, j) + min(i + lane, n - 1)];
                sum.tokens(a, at, min(n - i, 64), [&](int k) { return lane_value(more, k); });
            }
            sum.template put<GT>(a, at, row_of_block(j));
        }
    }
}

// Rows that were split: a block looks through kJoinWindows windows for those that start there, and sums a row's parts in order.  Rows
// of up to kJoinAlone parts take a wave each; for the others every wave sums a stretch and they meet in LDS.  Bound by latency: the most
// frequent row's parts, one after the other (65536 tokens of a vocabulary: 6.2 us, with 256 threads a block 8.8).
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64, kJoinWindows = 16, kJoinAlone = 8;
template <int GT, int N>
__global__ __launch_bounds__(kJoinThreads) void row_join_kernel(SumArgs a) {
    __shared__ float part[kJoinWaves][64 * N];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t window = static_cast<int64_t>(blockIdx.x) * kJoinWindows + lane;
    const uint32_t found = lane < kJoinWindows && window < a.windows ? a.split[window * 2 + 1] : 0u;
    const int parts_here = found != 0 ? static_cast<int>(((a.first[found] - 1) >> a.log2_window) - static_cast<uint32_t>(window)) + 1 : 0;
    SumArgs p = a;                                   // the parts as rows
    p.dout = reinterpret_cast<const char*>(a.partial);
    p.dout_stride = a.width;
    auto part_of = [&](int l, int i) { return (blockIdx.x * kJoinWindows + l + i) * 2 + (i == 0 ? 1u : 0u); };
    uint64_t few = __ballot(parts_here > 0 && parts_here <= kJoinAlone), many = __ballot(parts_here > kJoinAlone);
    for (int i = 0; few != 0; ++i, few &= few - 1) {
        if (i % kJoinWaves != wave) continue;
        const int l = __ffsll(static_cast<unsigned long long>(few)) - 1;
        const int parts = static_cast<int>(lane_value(parts_here, l));
        const int64_t row = row_at(a, lane_value(found, l) - 1);
        for (int c = blockIdx.y * (64 * N); c < a.width; c += gridDim.y * (64 * N)) {
            const Columns<N, 1> at(c, a.width);
            Sum<DDP_FP32, N, 1> sum;
            sum.tokens(p, at, parts, [&](int k) { return part_of(l, k); });
            sum.template put<GT>(a, at, row);
        }
    }
    for (; many != 0; many &= many - 1) {
        const int l = __ffsll(static_cast<unsigned long long>(many)) - 1;
        const int parts = static_cast<int>(lane_value(parts_here, l)), share = (parts + kJoinWaves - 1) / kJoinWaves;
        const int64_t row = row_at(a, lane_value(found, l) - 1);
        const int from = min(wave * share, parts), to = min(from + share, parts);
        for (int c = blockIdx.y * (64 * N); c < a.width; c += gridDim.y * (64 * N)) {
            const Columns<N, 1> at(c, a.width);
            Sum<DDP_FP32, N, 1> sum;
            sum.tokens(p, at, to - from, [&](int k) { return part_of(l, from + k); });
            if (wave > 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) part[wave][k * 64 + lane] = sum.acc[0][k];
            }
            __syncthreads();
            if (wave == 0) {
                for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                    for (int k = 0; k < N; ++k) sum.acc[0][k] += part[w][k * 64 + lane];
                sum.template put<GT>(a, at, row);
            }
            __syncthreads();
        }
    }
}

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

}  // namespace

struct ddp_embedding {
    int32_t device = DDP_DEVICE_NONE;
    hipStream_t stream = nullptr;
    int64_t rows = 0, width = 0, max_tokens = 0;
    int32_t bucket_bits = 0, shift = 0;          // 2^bucket_bits buckets of 2^shift rows
    char* mem = nullptr;                         // workspace of the gradient
    uint16_t* starts = nullptr;
    uint32_t *list = nullptr, *gathered = nullptr, *sorted = nullptr, *first = nullptr, *split = nullptr;
    float* partial = nullptr;
    std::string err;
};

namespace {

int32_t fail(ddp_embedding* e, int32_t code, const char* msg) {
    try {
        if (e) e->err = msg;
        else return ddp::fail_without_context(code, msg);
    } catch (...) {
    }
    return code;
}

#define EMB_HIP(e, expr)                                                            \
    do {                                                                            \
        const hipError_t e_ = taken(expr);                                          \
        if (e_ != hipSuccess) return fail((e), DDP_ERR_HIP, hipGetErrorString(e_)); \
    } while (0)

// Blocks of one column range each for the joins of a launch.
constexpr int kJoinRanges = 16;

template <typename Id, int WT, int OT>
void launch_lookup(ddp_embedding* e, int64_t tokens, const void* ids, const void* table, int64_t table_stride, float scale, void* out, int64_t out_stride) {
    constexpr int N = WT == DDP_FP32 || OT == DDP_FP32 ? 4 : 8;
    const dim3 grid(static_cast<unsigned>((tokens + kWaves - 1) / kWaves)), block(kThreads);
    const int stream = tokens * e->width * ElemBytes<OT>::value >= kStreamBytes;
    auto* const from = static_cast<const char*>(table);
    auto* const to = static_cast<char*>(out);
    const int width = static_cast<int>(e->width);
    if (width < N)
        hipLaunchKernelGGL((lookup_kernel<Id, WT, OT, 1>), grid, block, 0, e->stream, static_cast<const Id*>(ids), tokens, from, e->rows, width, table_stride,
                           scale, to, out_stride, stream);
    else if (width > 32 * N)
        hipLaunchKernelGGL((lookup_kernel<Id, WT, OT, N>), grid, block, 0, e->stream, static_cast<const Id*>(ids), tokens, from, e->rows, width, table_stride,
                           scale, to, out_stride, stream);
    else
        hipLaunchKernelGGL((narrow_lookup_kernel<Id, WT, OT, N>), dim3(static_cast<unsigned>((tokens * ((width + N - 1) / N) + kThreads - 1) / kThreads)), block, 0,
                           e->stream, static_cast<const Id*>(ids), static_cast<unsigned>(tokens), from, e->rows, width, table_stride, scale, to, out_stride, stream);
}
template <typename Id, typename... Rest>
void launch_lookup(int wt, int ot, Rest... rest) {
    switch (wt * 3 + ot) {
        case 0: return launch_lookup<Id, 0, 0>(rest...);
        case 1: return launch_lookup<Id, 0, 1>(rest...);
        case 2: return launch_lookup<Id, 0, 2>(rest...);
        case 3: return launch_lookup<Id, 1, 0>(rest...);
        case 4: return launch_lookup<Id, 1, 1>(rest...);
        case 5: return launch_lookup<Id, 1, 2>(rest...);
        case 6: return launch_lookup<Id, 2, 0>(rest...);
        case 7: return launch_lookup<Id, 2, 1>(rest...);
        default: return launch_lookup<Id, 2, 2>(rest...);
    }
}

template <typename Id, int FT, int GT, int N>
hipError_t launch_scan(ddp_embedding* e, SumArgs a) {
    a.units = static_cast<int32_t>((a.width + 64 * N - 1) / (64 * N));
    const int64_t blocks = std::min(int64_t(1) << a.log2_blocks, ((a.rows - 1) >> a.log2_run) + 1);
    const size_t counters = ((static_cast<size_t>(a.rows - 1) >> (a.log2_blocks + a.log2_run)) + 1) * (size_t(4) << a.log2_run);
    const int64_t bytes = a.width * (a.rows * ElemBytes<GT>::value + a.tokens * ElemBytes<FT>::value);
    const unsigned ranges = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>({a.units, kScanBlocks / blocks, bytes / (kScanBlockBytes * blocks)})));
    hipLaunchKernelGGL((scan_sum_kernel<Id, FT, GT, N>), dim3(static_cast<unsigned>(blocks), ranges), dim3(kScanThreads), counters, e->stream, a);
    return hipGetLastError();
}
template <int FT, int GT, int N, int WN>
hipError_t launch_rows(ddp_embedding* e, SumArgs a) {
    auto ranges_of = [&](int columns) { return static_cast<int32_t>((a.width + columns - 1) / columns); };
    a.units = ranges_of(64 * N);
    a.window_units = ranges_of(64 * WN);
    a.window_blocks = static_cast<int32_t>((static_cast<int64_t>(a.windows) * a.window_units + kWaves - 1) / kWaves);
    a.rows_per_block = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>({64, std::max(8, kRowColumns / a.width), a.rows / kRowBlocks})));
    a.row_blocks = static_cast<int32_t>((a.rows + a.rows_per_block - 1) / a.rows_per_block);
    const int64_t blocks = static_cast<int64_t>(a.window_blocks) + a.row_blocks;
    hipLaunchKernelGGL((row_sum_kernel<FT, GT, N, WN>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, e->stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    constexpr int JN = N == 1 ? 1 : 4;
    const int ranges = std::min(kJoinRanges, ranges_of(64 * JN));
    hipLaunchKernelGGL((row_join_kernel<GT, JN>), dim3(static_cast<unsigned>((a.windows + kJoinWindows - 1) / kJoinWindows), static_cast<unsigned>(ranges)),
                       dim3(kJoinThreads), 0, e->stream, a);
    return hipGetLastError();
}
template <typename Id, int FT, int GT>
hipError_t launch_sum(ddp_embedding* e, const SumArgs& a, bool scan) {
    constexpr int N = FT == DDP_FP32 || GT == DDP_FP32 ? 4 : 8;    // 16 bytes of the wider side: stores of whole lines
    constexpr int WN = FT == DDP_FP32 ? 4 : 8;
    if (a.width < WN) return scan ? launch_scan<Id, FT, GT, 1>(e, a) : launch_rows<FT, GT, 1, 1>(e, a);
    if (!scan) return launch_rows<FT, GT, N, WN>(e, a);
    return launch_scan<Id, FT, GT, N>(e, a);
}
template <typename Id>
hipError_t launch_sum(int ft, int gt, ddp_embedding* e, const SumArgs& a, bool scan) {
    switch (ft * 3 + gt) {
        case 0: return launch_sum<Id, 0, 0>(e, a, scan);
        case 1: return launch_sum<Id, 0, 1>(e, a, scan);
        case 2: return launch_sum<Id, 0, 2>(e, a, scan);
        case 3: return launch_sum<Id, 1, 0>(e, a, scan);
        case 4: return launch_sum<Id, 1, 1>(e, a, scan);
        case 5: return launch_sum<Id, 1, 2>(e, a, scan);
        case 6: return launch_sum<Id, 2, 0>(e, a, scan);
        case 7: return launch_sum<Id, 2, 1>(e, a, scan);
        default: return launch_sum<Id, 2, 2>(e, a, scan);
    }
}

template <typename Id>
hipError_t launch_sort(ddp_embedding* e, const SortArgs& a) {
    hipLaunchKernelGGL((chunk_sort_kernel<Id>), dim3(a.chunks), dim3(kChunk), static_cast<size_t>(a.buckets) * 4, e->stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(bucket_sort_kernel, dim3(a.buckets, a.shift == 0 && a.buckets <= 64 ? std::min(8, a.chunks) : 1), dim3(kSortThreads), (static_cast<size_t>(kSortWaves + 1) << a.shift) * 4, e->stream, a);
    return hipGetLastError();
}

bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

}  // namespace

extern "C" {

const char* ddp_embedding_last_error(const ddp_embedding* e) { return e ? e->err.c_str() : ddp_last_error(nullptr); }

int32_t ddp_embedding_create(ddp_embedding** out, int32_t device, void* stream, int64_t rows, int64_t width, int64_t max_tokens) {
    if (!out) return fail(nullptr, DDP_ERR_ARG, "ddp_embedding_create: out is null");
    *out = nullptr;
    if (device < DDP_DEVICE_NONE) return fail(nullptr, DDP_ERR_ARG, "ddp_embedding_create: bad device");
    if (rows < 1 || width < 1 || max_tokens < 0) return fail(nullptr, DDP_ERR_ARG, "ddp_embedding_create: rows and width are at least 1, max_tokens at least 0");
    if (rows > kMaxRows || width > kMaxWidth || max_tokens > kMaxTokens)
        return fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_embedding_create: more than 2^23 rows, 2^20 columns or 2^22 tokens");
    if (device != DDP_DEVICE_NONE) {
        int count = 0;
        if (taken(hipGetDeviceCount(&count)) != hipSuccess || device >= count)
            return fail(nullptr, DDP_ERR_HIP, "ddp_embedding_create: no such HIP device (the library needs a GPU; DDP_DEVICE_NONE checks arguments only)");
    }
    ddp_embedding* e = new (std::nothrow) ddp_embedding();
    if (!e) return fail(nullptr, DDP_ERR_HIP, "out of host memory");
    e->device = device;
    e->stream = static_cast<hipStream_t>(stream);
    e->rows = rows;
    e->width = width;
    e->max_tokens = max_tokens;
    // up to 1024 buckets, more where a bucket would have more than kSortRows rows
    while ((int64_t(1) << (e->bucket_bits + e->shift)) < rows) ++(e->bucket_bits < 10 || e->shift == 10 ? e->bucket_bits : e->shift);
    static_assert((kMaxRows >> 10) <= kMaxBuckets && (1 << 10) == kSortRows, "LDS of the sorting kernels");
    if (device != DDP_DEVICE_NONE && max_tokens > 0) {
        const int64_t chunks = (max_tokens + kChunk - 1) / kChunk;
        const int64_t places = int64_t(1) << (e->bucket_bits + e->shift), buckets = int64_t(1) << e->bucket_bits;
        const int64_t tokens = up(max_tokens * 4, 256), first = up((places + 1) * 4, 256), starts = up(chunks * (buckets + 1) * 2, 256);
        const int64_t split = up(chunks * (2 * kChunk >> kLog2Window) * 4, 256);
        const int64_t partial = (((max_tokens - 1) >> kLog2Window) + 1) * 2 * width * 4;
        hipError_t err = taken(hipSetDevice(device));
        if (err == hipSuccess) err = taken(hipMalloc(reinterpret_cast<void**>(&e->mem), 3 * tokens + first + split + up(partial, 256) + starts));
        if (err != hipSuccess) {
            delete e;
            return fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        char* at = e->mem;
        e->gathered = reinterpret_cast<uint32_t*>(at);
        e->list = reinterpret_cast<uint32_t*>(at += tokens);
        e->sorted = reinterpret_cast<uint32_t*>(at += tokens);
        e->first = reinterpret_cast<uint32_t*>(at += tokens);
        e->split = reinterpret_cast<uint32_t*>(at += first);
        e->partial = reinterpret_cast<float*>(at += split);
        e->starts = reinterpret_cast<uint16_t*>(at += up(partial, 256));
    }
    *out = e;
    return DDP_OK;
}

int32_t ddp_embedding_destroy(ddp_embedding* e) {
    if (!e) return DDP_ERR_ARG;
    if (e->device != DDP_DEVICE_NONE) {
        (void)taken(hipSetDevice(e->device));
        (void)taken(hipStreamSynchronize(e->stream));    // (lookups too: the caller frees what they use)
        if (e->mem) (void)taken(hipFree(e->mem));
    }
    delete e;
    return DDP_OK;
}

int32_t ddp_embedding_lookup(ddp_embedding* e, int64_t tokens, const void* ids, int32_t id_bits, const void* table, int32_t table_dtype,
                             int64_t table_stride, float scale, void* out, int32_t out_dtype, int64_t out_stride) {
    if (!e) return DDP_ERR_ARG;
    if (tokens < 0 || tokens > kMaxTokens) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: tokens outside [0, 2^22]");
    if (id_bits != 32 && id_bits != 64) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: ids have 32 or 64 bits");
    if (!known_dtype(table_dtype) || !known_dtype(out_dtype)) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: unknown dtype");
    if (table_stride < e->width || out_stride < e->width || table_stride > INT32_MAX || out_stride > INT32_MAX)
        return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: a stride is below the width (or above 2^31 - 1)");
    if (e->device == DDP_DEVICE_NONE) return fail(e, DDP_ERR_NO_DEVICE, "ddp_embedding_lookup without a device");
    if (tokens == 0) return DDP_OK;
    if (!ids || !table || !out) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: null pointer");
    if (misaligned(ids, id_bits / 8) || misaligned(table, elem_bytes(table_dtype)) || misaligned(out, elem_bytes(out_dtype)))
        return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: pointer not aligned to its element size");
    EMB_HIP(e, hipSetDevice(e->device));
    if (id_bits == 32) launch_lookup<int32_t>(table_dtype, out_dtype, e, tokens, ids, table, table_stride, scale, out, out_stride);
    else launch_lookup<int64_t>(table_dtype, out_dtype, e, tokens, ids, table, table_stride, scale, out, out_stride);
    EMB_HIP(e, hipGetLastError());
    return DDP_OK;
}

int32_t ddp_embedding_grad(ddp_embedding* e, int64_t tokens, const void* ids, int32_t id_bits, const void* dout, int32_t dout_dtype,
                           int64_t dout_stride, float scale, int64_t padding_row, int32_t accumulate, void* grad, int32_t grad_dtype, int64_t grad_stride) {
    if (!e) return DDP_ERR_ARG;
    if (tokens < 0 || tokens > e->max_tokens) return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: tokens outside [0, max_tokens]");
    if (id_bits != 32 && id_bits != 64) return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: ids have 32 or 64 bits");
    if (!known_dtype(dout_dtype) || !known_dtype(grad_dtype)) return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: unknown dtype");
    if (dout_stride < e->width || grad_stride < e->width || dout_stride > INT32_MAX || grad_stride > INT32_MAX)
        return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: a stride is below the width (or above 2^31 - 1)");
    if (padding_row < -1 || padding_row >= e->rows) return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: padding row outside the table (-1: none)");
    if (e->device == DDP_DEVICE_NONE) return fail(e, DDP_ERR_NO_DEVICE, "ddp_embedding_grad without a device");
    if (!grad || (tokens > 0 && (!ids || !dout))) return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: null pointer");
    if (misaligned(ids, id_bits / 8) || misaligned(dout, elem_bytes(dout_dtype)) || misaligned(grad, elem_bytes(grad_dtype)))
        return fail(e, DDP_ERR_ARG, "ddp_embedding_grad: pointer not aligned to its element size");
    EMB_HIP(e, hipSetDevice(e->device));
    if (!e->mem) return fail(e, DDP_ERR_STATE, "ddp_embedding_grad: the handle was made for no tokens");
    SumArgs a{};
    a.first = e->first;
    a.sorted = e->sorted;
    a.ids = ids;
    a.dout = static_cast<const char*>(dout);
    a.grad = static_cast<char*>(grad);
    a.partial = e->partial;
    a.split = e->split;
    a.tokens = tokens;
    a.rows = e->rows;
    a.width = static_cast<int32_t>(e->width);
    a.dout_stride = dout_stride;
    a.grad_stride = grad_stride;
    a.padding = padding_row;
    a.log2_window = log2_window(tokens, e->rows, (e->width * elem_bytes(dout_dtype) + 1023) / 1024);
    a.windows = static_cast<int32_t>((tokens + (1 << a.log2_window) - 1) >> a.log2_window);
    a.add = accumulate != 0;
    a.scale = scale;
    a.shift = e->shift;
    a.bucket_bits = e->bucket_bits;
    const int64_t each = std::min<int64_t>(1024, std::max<int64_t>(kScanRows, kScanRows * 1024 / e->width));
    while ((a.rows - 1) >> a.log2_blocks >= each) ++a.log2_blocks;
    while (a.log2_blocks < 9 && (int64_t(1) << a.log2_blocks) < a.rows) ++a.log2_blocks;
    if (a.log2_blocks > 9) {                         // enough rows to have them in pairs
        a.log2_run = 1;
        a.log2_blocks -= 1;
    }
    const bool scan = tokens <= std::min<int64_t>(kScanTokens, std::max<int64_t>(1024, 128 * e->rows));
    if (!scan) {
        SortArgs s{};
        s.ids = ids;
        s.tokens = tokens;
        s.rows = e->rows;
        s.padding = padding_row;
        s.shift = e->shift;
        s.buckets = 1 << e->bucket_bits;
        s.bucket_bits = e->bucket_bits;
        s.chunks = static_cast<int32_t>((tokens + kChunk - 1) / kChunk);
        s.starts = e->starts;
        s.list = e->list;
        s.gathered = e->gathered;
        s.sorted = e->sorted;
        s.first = e->first;
        s.split = e->split;
        s.log2_window = a.log2_window;
        EMB_HIP(e, id_bits == 32 ? launch_sort<int32_t>(e, s) : launch_sort<int64_t>(e, s));
    }
    EMB_HIP(e, id_bits == 32 ? launch_sum<int32_t>(dout_dtype, grad_dtype, e, a, scan) : launch_sum<int64_t>(dout_dtype, grad_dtype, e, a, scan));
    return DDP_OK;
}

}  // extern "C"
