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
constexpr int64_t kMaxRows = int64_t(1) << 23, kMaxTokens = int64_t(1) << 24, kMaxWidth = int64_t(1) << 20;

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

template <int DT, int N>
__device__ __forceinline__ void store_own(char* row, int at, int own, const float (&x)[N]) {
    char* to = row + at * ElemBytes<DT>::value;
    if (own == 0) {
        store_some<DT, N>(to, N, x);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= own) store_one<DT>(to + i * ElemBytes<DT>::value, x[i]);
    }
}
// N = 1 of a 16-bit type is half a dword: no vector access.
template <int DT, int N> struct Vector {
    Parts<DT, N> raw;
    __device__ __forceinline__ void load(const char* p) { raw = load_parts<DT, N>(p); }
    __device__ __forceinline__ void get(float (&x)[N]) const { widen<DT, N>(raw, x); }
};
template <int DT> struct Vector<DT, 1> {
    float x1;
    __device__ __forceinline__ void load(const char* p) { x1 = load_one<DT>(p); }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = x1; }
};
template <int DT>
__device__ __forceinline__ void store_own(char* row, int at, int own, const float (&x)[1]) {
    if (own == 0) store_one<DT>(row + at * ElemBytes<DT>::value, x[0]);
}

// ---- lookup ----

template <typename Id, int WT, int OT, int N>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const Id* ids, int64_t tokens, const char* table, int64_t rows, int width,
                                                          int64_t table_stride, float scale, char* out, int64_t out_stride) {
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
            store_own<OT>(to, at.at[s], at.own[s], x);
        }
    }
}

// ---- sums of tokens' rows ----

struct SumArgs {
    const uint32_t* first;
    const uint32_t* sorted;
    const void* ids;
    const char* dout;
    char* grad;
    float* partial;                              // [windows][2][width]
    int64_t tokens, rows, dout_stride, grad_stride, padding;
    int32_t width, window, windows, window_blocks, add;
    int32_t units, log2_blocks;                  // units: column ranges of a wave in a row
    float scale;
};

template <int FT, int N, int GROUPS>
struct Sum {
    // Tokens whose rows are on the way together: 16 KiB of a wave.
    static constexpr int U = N == 1 ? 8 : FT == DDP_FP32 ? 64 / (N * GROUPS) : 128 / (N * GROUPS);
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
    // The tokens that `token(i)` gives for i = 0 .. n-1, in this order; token(i) is the same in all lanes.
    template <typename Token>
    __device__ __forceinline__ void tokens(const SumArgs& a, const Columns<N, GROUPS>& at, int n, Token token) {
        int i = 0;
        for (; i + U <= n; i += U) several<U>(a, at, i, token);
        if constexpr (U > 4)
            for (; i + 4 <= n; i += 4) several<4>(a, at, i, token);
        if constexpr (U > 2)
            if (i + 2 <= n) { several<2>(a, at, i, token); i += 2; }
        for (; i < n; ++i) several<1>(a, at, i, token);
    }
    template <int K, typename Token>
    __device__ __forceinline__ void several(const SumArgs& a, const Columns<N, GROUPS>& at, int i, Token token) {
        Vector<FT, N> v[K][GROUPS];
#pragma unroll
        for (int u = 0; u < K; ++u) load(v[u], a, at, token(i + u));
#pragma unroll
        for (int u = 0; u < K; ++u) add(v[u], at);
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
                store_own<GT>(to, at.at[s], at.own[s], acc[s]);
            }
            return;
        }
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) {
            if (at.own[s] == N) continue;
#pragma unroll
            for (int k = 0; k < N; ++k) acc[s][k] *= a.scale;
            store_own<GT>(to, at.at[s], at.own[s], acc[s]);
        }
    }
};

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

// ---- few tokens: every block looks through all of them ----
//
// Block b of 2^log2_blocks has the rows b, b + blocks, ... (rows of frequent tokens are neighbours in many vocabularies: they go to
// different blocks).  It lists the tokens of its rows, t ascending, and its waves sum a row each; rows of many tokens
// are split over the block's waves and joined in LDS, in order.

constexpr int kScanThreads = 512, kScanWaves = kScanThreads / 64;
constexpr int kScanTokens = 4096;
constexpr int kScanEach = kScanTokens / kScanThreads;
constexpr int kScanAlone = 16;                   // tokens of a row that one wave sums
constexpr int kScanRows = 32;                    // rows of 1024 columns that a block has at most (up to 1024 of fewer columns)

template <typename Id, int FT, int GT, int N, int GROUPS>
__global__ __launch_bounds__(kScanThreads) void scan_sum_kernel(SumArgs a) {
    __shared__ uint32_t list[kScanTokens];           // row in the block << 16 | token
    __shared__ uint32_t wave_count[kScanWaves];
    __shared__ float part[kScanWaves][64 * N * GROUPS];
    extern __shared__ uint32_t crowded[];            // a bit for every row of the block that has many tokens
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.x;
    const int nrows = static_cast<int>((a.rows - b + (int64_t(1) << a.log2_blocks) - 1) >> a.log2_blocks);
    const int per_wave = static_cast<int>((a.tokens + kScanThreads - 1) / kScanThreads) * 64;
    for (int i = threadIdx.x; i < (nrows + 31) / 32; i += kScanThreads) crowded[i] = 0;
    int64_t row[kScanEach];
#pragma unroll
    for (int k = 0; k < kScanEach; ++k) {
        const int t = wave * per_wave + k * 64 + lane;
        row[k] = k * 64 < per_wave && t < a.tokens ? row_of(static_cast<const Id*>(a.ids), t) : -1;
    }
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < kScanEach; ++k) {
        if (row[k] < 0 || row[k] >= a.rows || row[k] == a.padding || (row[k] & ((int64_t(1) << a.log2_blocks) - 1)) != b) row[k] = -1;
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
        if (row[k] >= 0) list[next + lanes_below(hits)] = static_cast<uint32_t>(row[k] >> a.log2_blocks) << 16 | static_cast<uint32_t>(wave * per_wave + k * 64 + lane);
        next += __popcll(hits);
    }
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(static_cast<int>(listed));
    const int units = a.units;
    // rows of few tokens, a wave each
    for (int u = wave; u < nrows * units; u += kScanWaves) {
        const int j = u / units;
        int count = 0;
        for (int i = 0; i < n; i += 64) count += __popcll(__ballot(i + lane < n && list[min(i + lane, n - 1)] >> 16 == static_cast<uint32_t>(j)));
        if (count > kScanAlone) {
            if (lane == 0) atomicOr(&crowded[j >> 5], 1u << (j & 31));
            continue;
        }
        if (a.add && count == 0) continue;
        const Columns<N, GROUPS> at((u % units) * (64 * N * GROUPS), a.width);
        Sum<FT, N, GROUPS> sum;
        for (int i = 0; count > 0; i += 64) {
            const uint32_t e = list[min(i + lane, n - 1)];
            uint64_t hits = __ballot(i + lane < n && e >> 16 == static_cast<uint32_t>(j));
            const int here = __popcll(hits);
            count -= here;
            sum.tokens(a, at, here, [&](int) {
                const int l = __ffsll(static_cast<unsigned long long>(hits)) - 1;
                hits &= hits - 1;
                return lane_value(e, l) & 0xFFFFu;
            });
        }
        sum.template put<GT>(a, at, b + (static_cast<int64_t>(j) << a.log2_blocks));
    }
    __syncthreads();
    for (int j0 = 0; j0 < nrows; j0 += 32) {
        uint32_t bits = __builtin_amdgcn_readfirstlane(crowded[j0 >> 5]);
        while (bits != 0) {
            const int j = j0 + __ffs(bits) - 1;
            bits &= bits - 1;
            int count = 0;
            for (int i = 0; i < n; i += 64) count += __popcll(__ballot(i + lane < n && list[min(i + lane, n - 1)] >> 16 == static_cast<uint32_t>(j)));
            const int share = (count + kScanWaves - 1) / kScanWaves, from = wave * share, to = min(from + share, count);
            for (int unit = 0; unit < units; ++unit) {
                const Columns<N, GROUPS> at(unit * (64 * N * GROUPS), a.width);
                Sum<FT, N, GROUPS> sum;
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
#pragma unroll
                for (int s = 0; s < GROUPS; ++s)
#pragma unroll
                    for (int k = 0; k < N; ++k) part[wave][(s * N + k) * 64 + lane] = sum.acc[s][k];
                __syncthreads();
                if (wave == 0) {
#pragma unroll
                    for (int s = 0; s < GROUPS; ++s)
#pragma unroll
                        for (int k = 0; k < N; ++k)
                            for (int w = 1; w < kScanWaves; ++w) sum.acc[s][k] += part[w][(s * N + k) * 64 + lane];
                    sum.template put<GT>(a, at, b + (static_cast<int64_t>(j) << a.log2_blocks));
                }
                __syncthreads();
            }
        }
    }
}

// ---- more tokens: sorted by row ----
//
// Rows are put into buckets of 2^shift consecutive rows.  A block sorts a chunk of tokens by bucket; starts[chunk][b] is where
// bucket b starts in the chunk's part of `list`, which is also the number of the chunk's tokens in the buckets before it: summed
// over the chunks it is where the bucket starts among all tokens, so no scan over buckets is needed.  A block then
// gathers a bucket's tokens chunk by chunk (t ascending) and sorts them by row.

constexpr int kChunk = 1024;
constexpr int kMaxBuckets = 8192;                // 32 KiB of counters
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kSortRows = 1024;                  // rows of a bucket, at most
constexpr int kSortCache = 4096;                 // tokens of a bucket held in LDS

struct SortArgs {
    const void* ids;
    int64_t tokens, rows, padding;
    int32_t shift, buckets, bucket_bits, chunks;
    uint16_t* starts;                            // [chunks][buckets + 1]
    uint32_t* list;                              // [tokens] by chunk, by bucket: row in the bucket << 10 | token in the chunk
    uint64_t* gathered;                          // [tokens] by bucket, t ascending (buckets that LDS does not hold): row << 32 | token
    uint32_t* sorted;                            // [tokens] by row, t ascending
    uint32_t* first;                             // [rows + 1] where each row starts in `sorted`
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
    const uint32_t b = in ? static_cast<uint32_t>(row) >> a.shift : 0u;
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
    if (in) a.list[static_cast<int64_t>(blockIdx.x) * kChunk + count[b] + before + rank] = (static_cast<uint32_t>(row) & ((1u << a.shift) - 1)) << 10 | tid;
}

__global__ __launch_bounds__(kSortThreads) void bucket_sort_kernel(SortArgs a) {
    __shared__ uint64_t cache[kSortCache];
    __shared__ uint32_t wave_part[2][kSortWaves];
    __shared__ uint32_t more[kSortThreads], more_from[kSortThreads], more_to[kSortThreads];
    extern __shared__ uint32_t row_count[];          // [kSortWaves][rows of a bucket]
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = static_cast<int64_t>(b) << a.shift;
    const int nrows = static_cast<int>(min(static_cast<int64_t>(1) << a.shift, a.rows - row0));
    // where the bucket starts, and how many tokens it has
    uint32_t before = 0, mine = 0;
    for (int c = tid; c < a.chunks; c += kSortThreads) {
        const uint16_t* s = a.starts + static_cast<int64_t>(c) * (a.buckets + 1) + b;
        before += s[0];
        mine += s[1] - s[0];
    }
    const uint32_t before_all = wave_inclusive_sum(before), mine_all = wave_inclusive_sum(mine);
    if (lane == 63) {
        wave_part[0][wave] = before_all;
        wave_part[1][wave] = mine_all;
    }
    for (int i = tid; i < kSortWaves * nrows; i += kSortThreads) row_count[i] = 0;
    __syncthreads();
    uint32_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        base += wave_part[0][w];
        total += wave_part[1][w];
    }
    if (b == a.buckets - 1 && tid == 0) a.first[a.rows] = base + total;
    if (total == 0) {
        for (int r = tid; r < nrows; r += kSortThreads) a.first[row0 + r] = base;
        return;
    }
    // the bucket's tokens in order: a thread copies up to four of its chunk's, the waves together what there is above that
    uint64_t* tokens = total <= kSortCache ? cache : a.gathered + base;
    auto entry = [&](int c, uint32_t e) { return static_cast<uint64_t>(e >> 10) << 32 | (static_cast<uint32_t>(c) * kChunk + (e & (kChunk - 1))); };
    uint32_t done = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += kSortThreads) {
        const int c = c0 + tid;
        uint32_t s = 0, n = 0;
        if (c < a.chunks) {
            const uint16_t* p = a.starts + static_cast<int64_t>(c) * (a.buckets + 1) + b;
            s = p[0];
            n = p[1] - s;
        }
        const uint32_t upto = wave_inclusive_sum(n);
        __syncthreads();                             // wave_part and `more` are read by then
        if (lane == 63) wave_part[0][wave] = upto;
        __syncthreads();
        uint32_t to = done + upto - n;
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) to += wave_part[0][w];
            done += wave_part[0][w];
        }
        const uint32_t* from = a.list + static_cast<int64_t>(c) * kChunk + s;
        uint32_t few[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) few[i] = i < static_cast<int>(n) ? from[i] : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < static_cast<int>(n)) tokens[to + i] = entry(c, few[i]);
        more[tid] = n > 4 ? n - 4 : 0;
        more_from[tid] = s + 4;
        more_to[tid] = to + 4;
        const int rounds = min(kSortThreads, a.chunks - c0);
        if (!__syncthreads_or(n > 4)) continue;
        for (int k = wave; k < rounds; k += kSortWaves) {
            const uint32_t nk = __builtin_amdgcn_readfirstlane(more[k]);
            if (nk == 0) continue;
            const uint32_t* p = a.list + static_cast<int64_t>(c0 + k) * kChunk + more_from[k];
            uint64_t* q = tokens + more_to[k];
            for (uint32_t i0 = 0; i0 < nk; i0 += 256) {
                uint32_t e[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) e[u] = i0 + u * 64 + lane < nk ? p[i0 + u * 64 + lane] : 0u;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i0 + u * 64 + lane < nk) q[i0 + u * 64 + lane] = entry(c0 + k, e[u]);
            }
        }
    }
    __threadfence_block();
    __syncthreads();
    // counting sort by row: every wave has a stretch of the tokens
    const uint32_t stretch = (total + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
    const uint32_t from = min(wave * stretch, total), to = min(from + stretch, total);
    for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&row_count[wave * nrows + static_cast<uint32_t>(tokens[i] >> 32)], 1u);
    __syncthreads();
    // row by row, within a row wave by wave; the rows' sums are scanned in rounds of one row a thread
    uint32_t above = 0;
    for (int r0 = 0; r0 < nrows; r0 += kSortThreads) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < nrows)
            for (int w = 0; w < kSortWaves; ++w) n += row_count[w * nrows + r];
        const uint32_t upto = wave_inclusive_sum(n);
        if (lane == 63) wave_part[1][wave] = upto;
        __syncthreads();
        uint32_t next = above + upto - n;
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) next += wave_part[1][w];
            above += wave_part[1][w];
        }
        __syncthreads();
        if (r < nrows) {
            a.first[row0 + r] = base + next;
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t k = row_count[w * nrows + r];
                row_count[w * nrows + r] = next;
                next += k;
            }
        }
    }
    __syncthreads();
    uint32_t* place = row_count + wave * nrows;
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const uint32_t i = i0 + lane;
        const bool in = i < to;
        const uint64_t e = in ? tokens[i] : 0u;
        const uint32_t r = static_cast<uint32_t>(e >> 32);
        const uint64_t same = peers(r, a.shift, __ballot(in));
        const int rank = lanes_below(same);
        uint32_t p = 0;
        if (in) p = place[r];
        __builtin_amdgcn_wave_barrier();             // a wave's LDS accesses stay in order
        if (in) {
            a.sorted[base + p + rank] = static_cast<uint32_t>(e);
            if (rank == 0) place[r] = p + __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// A row of up to `window` tokens is summed by one wave (and column range); rows of more are split at multiples of `window`
// in the sorted tokens, their parts go through `partial` and are joined by another launch.
constexpr int kRowsPerBlock = 16;
constexpr int kWindow = 32;

// Window w's part of a row of more than `window` tokens: partial[w][0] where the row reaches back before the window, partial[w][1] where
// it starts in it (two such rows cannot start in one window).
template <typename Id, int FT, int N, int GROUPS>
__device__ __forceinline__ void sum_window(const SumArgs& a, int64_t w, int unit) {
    const uint32_t w0 = static_cast<uint32_t>(w) * a.window, all = a.first[a.rows];
    if (w0 >= all) return;
    const uint32_t w1 = min(w0 + a.window, all);
    const int64_t r_first = row_of(static_cast<const Id*>(a.ids), a.sorted[w0]), r_last = row_of(static_cast<const Id*>(a.ids), a.sorted[w1 - 1]);
    const Columns<N, GROUPS> at(unit * (64 * N * GROUPS), a.width);
    for (int side = 0; side < 2; ++side) {
        const int64_t r = side == 0 ? r_first : r_last;
        const uint32_t f = a.first[r], e = a.first[r + 1];
        if (e - f <= static_cast<uint32_t>(a.window) || (side == 0) != (f < w0)) continue;
        const uint32_t from = __builtin_amdgcn_readfirstlane(max(f, w0)), to = __builtin_amdgcn_readfirstlane(min(e, w1));
        Sum<FT, N, GROUPS> sum;
        for (uint32_t i = from; i < to; i += 64) {
            const uint32_t mine = a.sorted[min(i + (threadIdx.x & 63), to - 1)];
            sum.tokens(a, at, static_cast<int>(min(to - i, 64u)), [&](int k) { return lane_value(mine, k); });
        }
        char* p = reinterpret_cast<char*>(a.partial + (w * 2 + side) * static_cast<int64_t>(a.width));
#pragma unroll
        for (int s = 0; s < GROUPS; ++s)
            if (at.own[s] < N) store_own<DDP_FP32>(p, at.at[s], at.own[s], sum.acc[s]);
    }
}

// The first blocks take windows, the others kRowsPerBlock rows each: a row's sum, or zeros.
template <typename Id, int FT, int GT, int N, int GROUPS>
__global__ __launch_bounds__(kThreads) void row_sum_kernel(SumArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (static_cast<int>(blockIdx.x) < a.window_blocks) {
        const int64_t g = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
        if (g / a.units < a.windows) sum_window<Id, FT, N, GROUPS>(a, g / a.units, static_cast<int>(g % a.units));
        return;
    }
    const int64_t r0 = static_cast<int64_t>(static_cast<int>(blockIdx.x) - a.window_blocks) * kRowsPerBlock;
    const int nrows = static_cast<int>(min(static_cast<int64_t>(kRowsPerBlock), a.rows - r0));
    const uint32_t starts = a.first[r0 + min(lane, nrows)];
    const uint32_t block_from = lane_value(starts, 0), block_to = lane_value(starts, nrows);
    const uint32_t some = block_to > block_from ? a.sorted[min(block_from + lane, block_to - 1)] : 0u;      // the first 64 tokens
    for (int u = wave; u < nrows * a.units; u += kWaves) {
        const int j = u / a.units;
        const uint32_t from = lane_value(starts, j), to = lane_value(starts, j + 1);
        if (to - from > static_cast<uint32_t>(a.window) || (a.add && from == to)) continue;
        const Columns<N, GROUPS> at(u % a.units * (64 * N * GROUPS), a.width);
        Sum<FT, N, GROUPS> sum;
        if (to - block_from <= 64) {
            const int skip = static_cast<int>(from - block_from);
            sum.tokens(a, at, static_cast<int>(to - from), [&](int k) { return lane_value(some, skip + k); });
        } else {
            for (uint32_t i = from; i < to; i += 64) {
                const uint32_t mine = a.sorted[min(i + lane, to - 1)];
                sum.tokens(a, at, static_cast<int>(min(to - i, 64u)), [&](int k) { return lane_value(mine, k); });
            }
        }
        sum.template put<GT>(a, at, r0 + j);
    }
}

// A block for each window: where a row of more than `window` tokens starts in it, its parts are summed in order and written:
// a wave sums a stretch of them, the waves meet in LDS.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
template <typename Id, int GT, int N>
__global__ __launch_bounds__(kJoinThreads) void row_join_kernel(SumArgs a) {
    __shared__ float part[kJoinWaves][64 * N];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t w0 = blockIdx.x * a.window, all = a.first[a.rows];
    if (w0 >= all) return;
    const uint32_t w1 = min(w0 + a.window, all);
    const int64_t r = row_of(static_cast<const Id*>(a.ids), a.sorted[w1 - 1]);
    const uint32_t f = a.first[r], e = a.first[r + 1];
    if (e - f <= static_cast<uint32_t>(a.window) || f < w0) return;
    const int parts = static_cast<int>((e - 1) / a.window - blockIdx.x) + 1, share = (parts + kJoinWaves - 1) / kJoinWaves;
    const int from = min(wave * share, parts), to = min(from + share, parts);
    SumArgs p = a;                                   // the parts as rows: window blockIdx.x + i, its first half (the row's start: its second)
    p.dout = reinterpret_cast<const char*>(a.partial);
    p.dout_stride = a.width;
    for (int c = blockIdx.y * (64 * N); c < a.width; c += gridDim.y * (64 * N)) {
        const Columns<N, 1> at(c, a.width);
        Sum<DDP_FP32, N, 1> sum;
        sum.tokens(p, at, to - from, [&](int k) { return (blockIdx.x + from + k) * 2 + (from + k == 0 ? 1u : 0u); });
        if (wave > 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) part[wave][k * 64 + lane] = sum.acc[0][k];
        }
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                for (int k = 0; k < N; ++k) sum.acc[0][k] += part[w][k * 64 + lane];
            sum.template put<GT>(a, at, r);
        }
        __syncthreads();
    }
}

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

}  // namespace

struct ddp_embedding {
    int32_t device = DDP_DEVICE_NONE;
    hipStream_t stream = nullptr;
    int64_t rows = 0, width = 0, max_tokens = 0;
    int32_t shift = 0, buckets = 0;
    char* mem = nullptr;                         // workspace of the gradient
    uint16_t* starts = nullptr;
    uint64_t* gathered = nullptr;
    uint32_t *list = nullptr, *sorted = nullptr, *first = nullptr;
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
        const hipError_t e_ = (expr);                                               \
        if (e_ != hipSuccess) return fail((e), DDP_ERR_HIP, hipGetErrorString(e_)); \
    } while (0)

// Blocks of one column range each for the joins of a launch.
constexpr int kJoinRanges = 4;

template <typename Id, int WT, int OT>
void launch_lookup(ddp_embedding* e, int64_t tokens, const void* ids, const void* table, int64_t table_stride, float scale, void* out, int64_t out_stride) {
    constexpr int N = WT == DDP_FP32 || OT == DDP_FP32 ? 4 : 8;
    const dim3 grid(static_cast<unsigned>((tokens + kWaves - 1) / kWaves)), block(kThreads);
    if (e->width >= N)
        hipLaunchKernelGGL((lookup_kernel<Id, WT, OT, N>), grid, block, 0, e->stream, static_cast<const Id*>(ids), tokens,
                           static_cast<const char*>(table), e->rows, static_cast<int>(e->width), table_stride, scale, static_cast<char*>(out), out_stride);
    else
        hipLaunchKernelGGL((lookup_kernel<Id, WT, OT, 1>), grid, block, 0, e->stream, static_cast<const Id*>(ids), tokens,
                           static_cast<const char*>(table), e->rows, static_cast<int>(e->width), table_stride, scale, static_cast<char*>(out), out_stride);
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

template <typename Id, int FT, int GT, int N, int GROUPS>
hipError_t launch_scan(ddp_embedding* e, SumArgs a) {
    a.units = static_cast<int32_t>((a.width + 64 * N * GROUPS - 1) / (64 * N * GROUPS));
    const int64_t blocks = int64_t(1) << a.log2_blocks;
    const size_t flags = static_cast<size_t>(((a.rows >> a.log2_blocks) + 32) / 32) * 4;
    hipLaunchKernelGGL((scan_sum_kernel<Id, FT, GT, N, GROUPS>), dim3(static_cast<unsigned>(std::min(blocks, a.rows))), dim3(kScanThreads), flags, e->stream, a);
    return hipGetLastError();
}
template <typename Id, int FT, int GT, int N, int GROUPS>
hipError_t launch_rows(ddp_embedding* e, SumArgs a) {
    a.units = static_cast<int32_t>((a.width + 64 * N * GROUPS - 1) / (64 * N * GROUPS));
    a.window_blocks = static_cast<int32_t>((static_cast<int64_t>(a.windows) * a.units + kWaves - 1) / kWaves);
    const int64_t blocks = a.window_blocks + (a.rows + kRowsPerBlock - 1) / kRowsPerBlock;
    hipLaunchKernelGGL((row_sum_kernel<Id, FT, GT, N, GROUPS>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, e->stream, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.windows <= 1) return err;
    constexpr int JN = N == 1 ? 1 : 4;
    const int ranges = std::min(kJoinRanges, (a.width + 64 * JN - 1) / (64 * JN));
    hipLaunchKernelGGL((row_join_kernel<Id, GT, JN>), dim3(static_cast<unsigned>(a.windows), static_cast<unsigned>(ranges)), dim3(kJoinThreads), 0, e->stream, a);
    return hipGetLastError();
}
template <typename Id, int FT, int GT>
hipError_t launch_sum(ddp_embedding* e, const SumArgs& a, bool scan) {
    constexpr int N = FT == DDP_FP32 ? 4 : 8;
    if (a.width < N) return scan ? launch_scan<Id, FT, GT, 1, 1>(e, a) : launch_rows<Id, FT, GT, 1, 1>(e, a);
    return scan ? launch_scan<Id, FT, GT, N, 16 / N>(e, a) : launch_rows<Id, FT, GT, N, 16 / N>(e, a);
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
    hipLaunchKernelGGL(bucket_sort_kernel, dim3(a.buckets), dim3(kSortThreads), (static_cast<size_t>(kSortWaves) << a.shift) * 4, e->stream, a);
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
        return fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_embedding_create: more than 2^23 rows, 2^20 columns or 2^24 tokens");
    if (device != DDP_DEVICE_NONE) {
        int count = 0;
        if (hipGetDeviceCount(&count) != hipSuccess || device >= count)
            return fail(nullptr, DDP_ERR_HIP, "ddp_embedding_create: no such HIP device (the library needs a GPU; DDP_DEVICE_NONE checks arguments only)");
    }
    ddp_embedding* e = new (std::nothrow) ddp_embedding();
    if (!e) return fail(nullptr, DDP_ERR_HIP, "out of host memory");
    e->device = device;
    e->stream = static_cast<hipStream_t>(stream);
    e->rows = rows;
    e->width = width;
    e->max_tokens = max_tokens;
    while (e->shift < 10 && ((rows - 1) >> e->shift) + 1 > 1024) ++e->shift;
    e->buckets = static_cast<int32_t>(((rows - 1) >> e->shift) + 1);
    static_assert((kMaxRows >> 10) <= kMaxBuckets && (1 << 10) <= kSortRows, "LDS of the sorting kernels");
    if (device != DDP_DEVICE_NONE && max_tokens > 0) {
        const int64_t chunks = (max_tokens + kChunk - 1) / kChunk;
        const int64_t gathered = up(max_tokens * 8, 256), tokens = up(max_tokens * 4, 256), first = up((rows + 1) * 4, 256);
        const int64_t partial = up((max_tokens + kWindow - 1) / kWindow * 2 * width * 4, 256), starts = up(chunks * (e->buckets + 1) * 2, 256);
        hipError_t err = hipSetDevice(device);
        if (err == hipSuccess) err = hipMalloc(reinterpret_cast<void**>(&e->mem), gathered + 2 * tokens + first + partial + starts);
        if (err != hipSuccess) {
            delete e;
            return fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        char* at = e->mem;
        e->gathered = reinterpret_cast<uint64_t*>(at);
        e->list = reinterpret_cast<uint32_t*>(at += gathered);
        e->sorted = reinterpret_cast<uint32_t*>(at += tokens);
        e->first = reinterpret_cast<uint32_t*>(at += tokens);
        e->partial = reinterpret_cast<float*>(at += first);
        e->starts = reinterpret_cast<uint16_t*>(at += partial);
    }
    *out = e;
    return DDP_OK;
}

int32_t ddp_embedding_destroy(ddp_embedding* e) {
    if (!e) return DDP_ERR_ARG;
    if (e->mem) {
        (void)hipSetDevice(e->device);
        (void)hipStreamSynchronize(e->stream);
        (void)hipFree(e->mem);
    }
    delete e;
    return DDP_OK;
}

int32_t ddp_embedding_lookup(ddp_embedding* e, int64_t tokens, const void* ids, int32_t id_bits, const void* table, int32_t table_dtype,
                             int64_t table_stride, float scale, void* out, int32_t out_dtype, int64_t out_stride) {
    if (!e) return DDP_ERR_ARG;
    if (tokens < 0 || tokens > kMaxTokens) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: tokens outside [0, 2^24]");
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
    a.tokens = tokens;
    a.rows = e->rows;
    a.width = static_cast<int32_t>(e->width);
    a.dout_stride = dout_stride;
    a.grad_stride = grad_stride;
    a.padding = padding_row;
    a.window = kWindow;
    a.windows = static_cast<int32_t>((tokens + a.window - 1) / a.window);
    a.add = accumulate != 0;
    a.scale = scale;
    const int64_t each = std::min<int64_t>(1024, std::max<int64_t>(kScanRows, kScanRows * 1024 / e->width));
    while ((a.rows - 1) >> a.log2_blocks >= each) ++a.log2_blocks;
    while (a.log2_blocks < 9 && (int64_t(1) << a.log2_blocks) < a.rows) ++a.log2_blocks;
    const bool scan = tokens <= kScanTokens;
    if (!scan) {
        SortArgs s{};
        s.ids = ids;
        s.tokens = tokens;
        s.rows = e->rows;
        s.padding = padding_row;
        s.shift = e->shift;
        s.buckets = e->buckets;
        while ((1 << s.bucket_bits) < s.buckets) ++s.bucket_bits;
        s.chunks = static_cast<int32_t>((tokens + kChunk - 1) / kChunk);
        s.starts = e->starts;
        s.list = e->list;
        s.gathered = e->gathered;
        s.sorted = e->sorted;
        s.first = e->first;
        EMB_HIP(e, id_bits == 32 ? launch_sort<int32_t>(e, s) : launch_sort<int64_t>(e, s));
    }
    EMB_HIP(e, id_bits == 32 ? launch_sum<int32_t>(dout_dtype, grad_dtype, e, a, scan) : launch_sum<int64_t>(dout_dtype, grad_dtype, e, a, scan));
    return DDP_OK;
}

}  // extern "C"
