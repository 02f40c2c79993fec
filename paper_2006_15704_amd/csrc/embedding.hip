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
constexpr int64_t kMaxRows = int64_t(1) << 23, kMaxTokens = int64_t(1) << 26, kMaxWidth = int64_t(1) << 20;

template <typename Id>
__device__ __forceinline__ int64_t row_of(const Id* ids, int64_t t) { return static_cast<int64_t>(*(DDP_GLOBAL_MEM const Id*)(ids + t)); }

// ---- lookup ----

template <typename Id, int WT, int OT>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const Id* ids, int64_t tokens, const char* table, int64_t rows, int64_t width,
                                                          int64_t table_stride, float scale, char* out, int64_t out_stride) {
    constexpr int N = WT == DDP_FP32 || OT == DDP_FP32 ? 4 : 8;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (t >= tokens) return;
    const int64_t r = row_of(ids, t);
    const bool named = r >= 0 && r < rows;
    const char* from = table + (named ? r : 0) * table_stride * ElemBytes<WT>::value;
    char* to = out + t * out_stride * ElemBytes<OT>::value;
    for (int64_t c = (threadIdx.x & 63) * N; c < width; c += 64 * N) {
        const int have = width - c >= N ? N : static_cast<int>(width - c);
        float x[N];
        load_some<WT, N>(from + c * ElemBytes<WT>::value, named ? have : 0, x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= scale;
        store_some<OT, N>(to + c * ElemBytes<OT>::value, have, x);
    }
}

// ---- sorting the tokens by row ----
//
// Rows are put into buckets of 2^shift consecutive rows.  A wave sorts a chunk of tokens by bucket; starts[chunk][b] is where
// bucket b starts in the chunk's part of `list`, which is also the number of the chunk's tokens in the buckets before it: summed
// over the chunks it is where the bucket starts among all tokens, so no scan over buckets is needed.  A block then
// gathers a bucket's tokens chunk by chunk (t ascending) and sorts them by row.

constexpr int kMaxBuckets = 8192;                // 33 KiB of counters
constexpr int kMinChunk = 1024, kMaxChunks = 4096;
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kSortRows = 1024;                  // rows of a bucket, at most
constexpr int kSortCache = 4096;                 // tokens of a bucket held in LDS

struct SortArgs {
    const void* ids;
    int64_t tokens, rows, padding;
    int32_t shift, buckets, chunk, chunks;
    uint32_t* starts;                            // [chunks][buckets + 1]
    uint32_t* list;                              // [tokens] by chunk, by bucket
    uint32_t* gathered;                          // [tokens] by bucket, t ascending (buckets that LDS does not hold)
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

// The token's row, or -1 where it takes no part.
template <typename Id>
__device__ __forceinline__ int32_t counted_row(const SortArgs& a, int64_t t) {
    const int64_t r = row_of(static_cast<const Id*>(a.ids), t);
    return r >= 0 && r < a.rows && r != a.padding ? static_cast<int32_t>(r) : -1;
}

template <typename Id>
__global__ __launch_bounds__(64) void chunk_sort_kernel(SortArgs a) {
    extern __shared__ uint32_t count[];              // [buckets], one word in 64 left out: lanes scan runs of 64 buckets
    auto at = [](int b) { return b + (b >> 6); };
    const int lane = threadIdx.x;
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.chunk;
    const int here = static_cast<int>(min(static_cast<int64_t>(a.chunk), a.tokens - t0));
    for (int i = lane; i < at(a.buckets) + 1; i += 64) count[i] = 0;
    __syncthreads();
    for (int i = lane; i < here; i += 64) {
        const int32_t r = counted_row<Id>(a, t0 + i);
        if (r >= 0) atomicAdd(&count[at(r >> a.shift)], 1u);
    }
    __syncthreads();
    // exclusive scan: a lane sums a run of buckets, the lanes' sums are scanned
    const int run = (a.buckets + 63) >> 6;
    const int from = min(lane * run, a.buckets), to = min(from + run, a.buckets);
    uint32_t sum = 0;
    for (int b = from; b < to; ++b) sum += count[at(b)];
    const uint32_t upto = wave_inclusive_sum(sum);
    uint32_t next = upto - sum;
    uint32_t* starts = a.starts + static_cast<int64_t>(blockIdx.x) * (a.buckets + 1);
    for (int b = from; b < to; ++b) {
        const uint32_t n = count[at(b)];
        count[at(b)] = next;
        next += n;
    }
    __syncthreads();
    for (int b = lane; b < a.buckets; b += 64) starts[b] = count[at(b)];
    if (lane == 63) starts[a.buckets] = upto;
    __syncthreads();
    const int bits = a.buckets > 1 ? 32 - __clz(a.buckets - 1) : 0;
    for (int i0 = 0; i0 < here; i0 += 64) {
        const int i = i0 + lane;
        const int32_t r = i < here ? counted_row<Id>(a, t0 + i) : -1;
        const uint32_t b = r < 0 ? 0u : static_cast<uint32_t>(r) >> a.shift;
        const uint64_t same = peers(b, bits, __ballot(r >= 0));
        const int rank = lanes_below(same);
        uint32_t place = 0;
        if (r >= 0) place = count[at(b)];
        __syncthreads();                             // (one wave: orders the reads before the writes)
        if (r >= 0) {
            a.list[t0 + place + rank] = static_cast<uint32_t>(t0 + i);
            if (rank == 0) count[at(b)] = place + __popcll(same);
        }
        __syncthreads();
    }
}

template <typename Id>
__global__ __launch_bounds__(kSortThreads) void bucket_sort_kernel(SortArgs a) {
    __shared__ uint32_t cache[kSortCache];
    __shared__ uint32_t wave_part[2][kSortWaves];
    extern __shared__ uint32_t row_count[];          // [kSortWaves][rows of a bucket]
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = static_cast<int64_t>(b) << a.shift;
    const int nrows = static_cast<int>(min(static_cast<int64_t>(1) << a.shift, a.rows - row0));
    // where the bucket starts, and how many tokens it has
    uint32_t before = 0, mine = 0;
    for (int c = tid; c < a.chunks; c += kSortThreads) {
        const uint32_t* s = a.starts + static_cast<int64_t>(c) * (a.buckets + 1) + b;
        before += s[0];
        mine += s[1] - s[0];
    }
    uint32_t before_all = wave_inclusive_sum(before), mine_all = wave_inclusive_sum(mine);
    if (lane == 63) {
        wave_part[0][wave] = before_all;
        wave_part[1][wave] = mine_all;
    }
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
    // the bucket's tokens in order, chunk by chunk
    uint32_t* tokens = total <= kSortCache ? cache : a.gathered + base;
    uint32_t done = 0;
    for (int c0 = 0; c0 < a.chunks; c0 += kSortThreads) {
        const int c = c0 + tid;
        uint32_t s = 0, n = 0;
        if (c < a.chunks) {
            const uint32_t* p = a.starts + static_cast<int64_t>(c) * (a.buckets + 1) + b;
            s = p[0];
            n = p[1] - s;
        }
        const uint32_t upto = wave_inclusive_sum(n);
        __syncthreads();                             // wave_part is read by then
        if (lane == 63) wave_part[0][wave] = upto;
        __syncthreads();
        uint32_t to = done + upto - n;
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) to += wave_part[0][w];
            done += wave_part[0][w];
        }
        const uint32_t* from = a.list + static_cast<int64_t>(c) * a.chunk + s;
        for (uint32_t i = 0; i < n; ++i) tokens[to + i] = from[i];
    }
    // counting sort by row: every wave has a stretch of the tokens
    for (int i = tid; i < kSortWaves * nrows; i += kSortThreads) row_count[i] = 0;
    __threadfence_block();
    __syncthreads();
    const uint32_t stretch = (total + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
    const uint32_t from = min(wave * stretch, total), to = min(from + stretch, total);
    for (uint32_t i = from + lane; i < to; i += 64)
        atomicAdd(&row_count[wave * nrows + (counted_row<Id>(a, tokens[i]) - static_cast<int32_t>(row0))], 1u);
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
        const uint32_t t = in ? tokens[i] : 0u;
        const uint32_t r = in ? static_cast<uint32_t>(counted_row<Id>(a, t) - static_cast<int32_t>(row0)) : 0u;
        const uint64_t same = peers(r, a.shift, __ballot(in));
        const int rank = lanes_below(same);
        uint32_t p = 0;
        if (in) p = place[r];
        __builtin_amdgcn_wave_barrier();             // a wave's LDS accesses stay in order
        if (in) {
            a.sorted[base + p + rank] = t;
            if (rank == 0) place[r] = p + __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- sums by row ----

constexpr int kCold = 32;                        // tokens of a row that one wave sums; more are split over windows of as many
constexpr int kRowsPerBlock = 16;

struct SumArgs {
    const uint32_t* first;
    const uint32_t* sorted;
    const void* ids;
    const char* dout;
    char* grad;
    float* partial;                              // [windows][2][width]
    int64_t rows, width, dout_stride, grad_stride;
    int32_t windows, add;
    float scale;
};

// Elements of a lane in a slice: 16 bytes of what is read.
template <int FT> struct Lane { static constexpr int N = FT == DDP_FP32 ? 4 : 8; };

// acc += dout[t, c .. c + have) over tokens[from .. to), in this order.
template <int FT, int N>
__device__ __forceinline__ void sum_tokens(const SumArgs& a, const uint32_t* tokens, uint32_t from, uint32_t to, int64_t c, int have, float (&acc)[N]) {
    constexpr int B = ElemBytes<FT>::value, U = 8;
    for (uint32_t i = from; i < to; i += U) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = i + u < to;
            const uint32_t t = tokens[in ? i + u : to - 1];
            load_some<FT, N>(a.dout + (static_cast<int64_t>(t) * a.dout_stride + c) * B, in ? have : 0, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += x[u][k];
    }
}

template <int GT, int N>
__device__ __forceinline__ void put_row(const SumArgs& a, int64_t r, int64_t c, int have, float (&acc)[N]) {
    char* to = a.grad + (r * a.grad_stride + c) * ElemBytes<GT>::value;
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] *= a.scale;
    if (a.add) {
        float old[N];
        load_some<GT, N>(to, have, old);
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] += old[k];
    }
    store_some<GT, N>(to, have, acc);
}

// Blocks 0 .. windows-1: the part of rows with more than kCold tokens that lies in window w of the sorted tokens,
// into partial[w][0] (the row reaches back before the window) or partial[w][1] (it starts in it; two such rows cannot start in
// one window).  Blocks from there on: rows with fewer tokens, summed and written, and rows without any, zeroed.
template <typename Id, int FT, int GT>
__global__ __launch_bounds__(kThreads) void row_sum_kernel(SumArgs a) {
    constexpr int N = Lane<FT>::N;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slices = static_cast<int>((a.width + 64 * N - 1) / (64 * N));
    if (static_cast<int>(blockIdx.x) < a.windows) {
        const uint32_t w0 = blockIdx.x * kCold, all = a.first[a.rows];
        if (w0 >= all) return;
        const uint32_t w1 = min(w0 + kCold, all);
        // the first row that starts in or before the window, and the one that the window ends in
        const int64_t r_first = row_of(static_cast<const Id*>(a.ids), a.sorted[w0]), r_last = row_of(static_cast<const Id*>(a.ids), a.sorted[w1 - 1]);
        for (int side = 0; side < 2; ++side) {
            const int64_t r = side == 0 ? r_first : r_last;
            const uint32_t f = a.first[r], e = a.first[r + 1];
            if (e - f <= kCold || (side == 0) != (f < w0)) continue;
            const uint32_t from = max(f, w0), to = min(e, w1);
            for (int s = wave; s < slices; s += kWaves) {
                const int64_t c = (static_cast<int64_t>(s) * 64 + lane) * N;
                const int have = a.width - c >= N ? N : a.width > c ? static_cast<int>(a.width - c) : 0;
                float acc[N] = {};
                sum_tokens<FT, N>(a, a.sorted, from, to, c, have, acc);
                float* p = a.partial + (static_cast<int64_t>(blockIdx.x) * 2 + side) * a.width + c;
                store_some<DDP_FP32, N>(p, have, acc);
            }
        }
        return;
    }
    const int64_t r0 = static_cast<int64_t>(blockIdx.x - a.windows) * kRowsPerBlock;
    const int nrows = static_cast<int>(min(static_cast<int64_t>(kRowsPerBlock), a.rows - r0));
    for (int u = wave; u < nrows * slices; u += kWaves) {
        const int64_t r = r0 + u / slices;
        const int64_t c = (static_cast<int64_t>(u % slices) * 64 + lane) * N;
        const int have = a.width - c >= N ? N : a.width > c ? static_cast<int>(a.width - c) : 0;
        const uint32_t from = a.first[r], to = a.first[r + 1];
        if (to - from > kCold || (a.add && from == to)) continue;
        float acc[N] = {};
        sum_tokens<FT, N>(a, a.sorted, from, to, c, have, acc);
        put_row<GT, N>(a, r, c, have, acc);
    }
}

// A block for each window: where a row of more than kCold tokens starts in it, its parts are summed in order and written.
template <typename Id, int GT>
__global__ __launch_bounds__(kThreads) void row_join_kernel(SumArgs a) {
    constexpr int N = 4;
    const uint32_t w0 = blockIdx.x * kCold, all = a.first[a.rows];
    if (w0 >= all) return;
    const uint32_t w1 = min(w0 + kCold, all);
    const int64_t r = row_of(static_cast<const Id*>(a.ids), a.sorted[w1 - 1]);
    const uint32_t f = a.first[r], e = a.first[r + 1];
    if (e - f <= kCold || f < w0) return;
    const uint32_t last = (e - 1) / kCold;
    for (int64_t c = threadIdx.x * N; c < a.width; c += kThreads * N) {
        const int have = a.width - c >= N ? N : static_cast<int>(a.width - c);
        float acc[N];
        load_some<DDP_FP32, N>(a.partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * a.width + c, have, acc);
        for (uint32_t w = blockIdx.x + 1; w <= last; ++w) {
            float x[N];
            load_some<DDP_FP32, N>(a.partial + static_cast<int64_t>(w) * 2 * a.width + c, have, x);
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] += x[k];
        }
        put_row<GT, N>(a, r, c, have, acc);
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
    uint32_t *starts = nullptr, *list = nullptr, *gathered = nullptr, *sorted = nullptr, *first = nullptr;
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

int32_t chunk_of(int64_t tokens) {
    return static_cast<int32_t>(std::max<int64_t>(kMinChunk, up((tokens + kMaxChunks - 1) / kMaxChunks, 64)));
}

template <typename Id, int WT, int OT>
void launch_lookup(ddp_embedding* e, int64_t tokens, const void* ids, const void* table, int64_t table_stride, float scale, void* out, int64_t out_stride) {
    const int64_t blocks = (tokens + kWaves - 1) / kWaves;
    hipLaunchKernelGGL((lookup_kernel<Id, WT, OT>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, e->stream, static_cast<const Id*>(ids), tokens,
                       static_cast<const char*>(table), e->rows, e->width, table_stride, scale, static_cast<char*>(out), out_stride);
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

template <typename Id, int FT, int GT>
void launch_sum(ddp_embedding* e, const SumArgs& a) {
    const int64_t blocks = a.windows + (a.rows + kRowsPerBlock - 1) / kRowsPerBlock;
    hipLaunchKernelGGL((row_sum_kernel<Id, FT, GT>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, e->stream, a);
    if (a.windows > 1) hipLaunchKernelGGL((row_join_kernel<Id, GT>), dim3(static_cast<unsigned>(a.windows)), dim3(kThreads), 0, e->stream, a);
}
template <typename Id>
void launch_sum(int ft, int gt, ddp_embedding* e, const SumArgs& a) {
    switch (ft * 3 + gt) {
        case 0: return launch_sum<Id, 0, 0>(e, a);
        case 1: return launch_sum<Id, 0, 1>(e, a);
        case 2: return launch_sum<Id, 0, 2>(e, a);
        case 3: return launch_sum<Id, 1, 0>(e, a);
        case 4: return launch_sum<Id, 1, 1>(e, a);
        case 5: return launch_sum<Id, 1, 2>(e, a);
        case 6: return launch_sum<Id, 2, 0>(e, a);
        case 7: return launch_sum<Id, 2, 1>(e, a);
        default: return launch_sum<Id, 2, 2>(e, a);
    }
}

template <typename Id>
hipError_t launch_sort(ddp_embedding* e, const SortArgs& a) {
    const size_t counters = (static_cast<size_t>(a.buckets) + a.buckets / 64 + 2) * 4;
    hipLaunchKernelGGL((chunk_sort_kernel<Id>), dim3(a.chunks), dim3(64), counters, e->stream, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const size_t row_counters = (static_cast<size_t>(kSortWaves) << a.shift) * 4;
    hipLaunchKernelGGL((bucket_sort_kernel<Id>), dim3(a.buckets), dim3(kSortThreads), row_counters, e->stream, a);
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
        return fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_embedding_create: more than 2^23 rows, 2^20 columns or 2^26 tokens");
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
        const int64_t chunks = (max_tokens + kMinChunk - 1) / kMinChunk;
        const int64_t starts = up(std::min<int64_t>(chunks, kMaxChunks) * (e->buckets + 1) * 4, 256);
        const int64_t tokens = up(max_tokens * 4, 256), first = up((rows + 1) * 4, 256);
        const int64_t partial = up((max_tokens + kCold - 1) / kCold * 2 * width * 4, 256);
        hipError_t err = hipSetDevice(device);
        if (err == hipSuccess) err = hipMalloc(reinterpret_cast<void**>(&e->mem), starts + 3 * tokens + first + partial);
        if (err != hipSuccess) {
            delete e;
            return fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        e->starts = reinterpret_cast<uint32_t*>(e->mem);
        e->list = reinterpret_cast<uint32_t*>(e->mem + starts);
        e->gathered = reinterpret_cast<uint32_t*>(e->mem + starts + tokens);
        e->sorted = reinterpret_cast<uint32_t*>(e->mem + starts + 2 * tokens);
        e->first = reinterpret_cast<uint32_t*>(e->mem + starts + 3 * tokens);
        e->partial = reinterpret_cast<float*>(e->mem + starts + 3 * tokens + first);
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
    if (tokens < 0 || tokens > kMaxTokens) return fail(e, DDP_ERR_ARG, "ddp_embedding_lookup: tokens outside [0, 2^26]");
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
    SortArgs s{};
    s.ids = ids;
    s.tokens = tokens;
    s.rows = e->rows;
    s.padding = padding_row;
    s.shift = e->shift;
    s.buckets = e->buckets;
    s.chunk = chunk_of(tokens);
    s.chunks = static_cast<int32_t>(std::max<int64_t>(1, (tokens + s.chunk - 1) / s.chunk));
    s.starts = e->starts;
    s.list = e->list;
    s.gathered = e->gathered;
    s.sorted = e->sorted;
    s.first = e->first;
    EMB_HIP(e, id_bits == 32 ? launch_sort<int32_t>(e, s) : launch_sort<int64_t>(e, s));
    SumArgs a{};
    a.first = e->first;
    a.sorted = e->sorted;
    a.ids = ids;
    a.dout = static_cast<const char*>(dout);
    a.grad = static_cast<char*>(grad);
    a.partial = e->partial;
    a.rows = e->rows;
    a.width = e->width;
    a.dout_stride = dout_stride;
    a.grad_stride = grad_stride;
    a.windows = static_cast<int32_t>((tokens + kCold - 1) / kCold);
    a.add = accumulate != 0;
    a.scale = scale;
    if (id_bits == 32) launch_sum<int32_t>(dout_dtype, grad_dtype, e, a);
    else launch_sum<int64_t>(dout_dtype, grad_dtype, e, a);
    EMB_HIP(e, hipGetLastError());
    return DDP_OK;
}

}  // extern "C"
