// Learned relative position bias by buckets, and its gradient.
//
//   r = key position - query position = j - i - offset
//   f(d) = d for d < exact, else min(n - 1, exact + floor((n - exact) log(d / exact) / log(distance / exact)))
//   bucket(r) = f(max(-r, 0)) with n = buckets, or with both directions n = buckets / 2: f(|r|), + n for r > 0
//   out[b, h, i, j]  = scale table[bucket(j - i - offset)][h]  (+ what is there)
//   grad[k][h]       = scale (sum of dscores[b, h, i, j] over the visible places of bucket k)  (+ what is there)
//
// A bias depends on the diagonal alone: forward is a fill, backward a sum along diagonals.  Both are bound by memory: 16 x 4096 x 4096 causal
// bfloat16 scores (537 MB) are filled in 91 us, 5.9 TB/s (a plain fill of as many bytes 78); the gradient of 2 x 16 x 4096 x 4096 (537 MB visible)
// takes 98, of which 93 read 590 MB at 6.3 TB/s; 8 x 16 x 512 x 512 binary32 of ragged lengths 21.8, the join 4 of them.
#include "extent.h"
#include "layer_host.h"

#include <cmath>
#include <vector>

struct ddp_position_bias : ddp::LayerHandle {
    int32_t heads = 0, buckets = 0, exact = 0, both = 0, sides = 0;      // sides: buckets of one direction
    int64_t distance = 0;
    int32_t parts = 0;                           // of the gradient that the workspace holds
    int32_t* first = nullptr;                    // [sides] the smallest distance of each bucket
    float* partial = nullptr;                    // [parts][heads][buckets]
    std::vector<int32_t> first_host;
};

namespace {

using namespace ddp;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxBuckets = 1024, kMaxHeads = 4096;
constexpr int64_t kFar = int64_t(1) << 40;
constexpr int64_t kMaxDistance = int64_t(1) << 20, kMaxLength = int64_t(1) << 24, kMaxBatch = int64_t(1) << 20;

// Whole numbers of any size: what a logarithm's step at exactly a whole distance takes to be settled.
struct Big {
    std::vector<uint32_t> w{1};
    void times(uint32_t x) {
        uint64_t carry = 0;
        for (uint32_t& d : w) {
            carry += static_cast<uint64_t>(d) * x;
            d = static_cast<uint32_t>(carry);
            carry >>= 32;
        }
        if (carry) w.push_back(static_cast<uint32_t>(carry));
    }
    void times_power(uint32_t x, int n) {
        for (int i = 0; i < n; ++i) times(x);
    }
    bool at_least(const Big& o) const {
        if (w.size() != o.w.size()) return w.size() > o.w.size();
        for (size_t i = w.size(); i-- > 0;)
            if (w[i] != o.w[i]) return w[i] > o.w[i];
        return true;
    }
};

// The smallest whole d with m log(d / e) / log(far / e) >= t, that is d^m >= e^(m - t) far^t.  Where the root is not near a whole
// number its rounding decides nothing; where it is, the powers are compared.
int32_t first_distance(int32_t e, int64_t far, int t, int m) {
    if (t == 0) return e;
    const long double root = e * std::pow(static_cast<long double>(far) / e, static_cast<long double>(t) / m);
    const long double near = std::floor(root + 0.5L);
    if (std::fabs(root - near) > 1e-10L * root) return static_cast<int32_t>(std::ceil(root));
    Big d, want;
    d.times_power(static_cast<uint32_t>(near), m);
    want.times_power(static_cast<uint32_t>(e), m - t);
    want.times_power(static_cast<uint32_t>(far), t);
    return static_cast<int32_t>(near) + (d.at_least(want) ? 0 : 1);
}

struct BiasArgs {
    const int32_t *first, *key_lengths, *query_lengths;
    const char* table;
    char* scores;                                // dscores in the gradient
    float* partial;
    int64_t batch, queries, keys, offset, table_stride, s_batch, s_head, s_query;
    int64_t band0, last, strips, center;         // of the gradient: the first lane of the first strip, the last that is visible
    int64_t tiles, plane_tiles, col_tiles;       // of the bias
    int32_t heads, buckets, sides, both, causal, strip_blocks, shares, rows, cols, log2_cols, regions;
    float scale, masked;
};

__device__ __forceinline__ int bucket_of(const int32_t* first, const BiasArgs& a, int64_t r) {
    const int64_t d = a.both ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
    int lo = 0, hi = a.sides;                        // first[lo] <= d < first[hi]
    if (d >= first[hi - 1]) lo = hi - 1;             // (most diagonals of long scores)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= d) lo = mid;
        else hi = mid;
    }
    return lo + (a.both && r > 0 ? a.sides : 0);
}
__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t b, int64_t most) {
    if (lengths == nullptr) return most;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n < most ? n : most;
}

// ---- bias ----
//
// A block has `cols` vectors of N keys side by side and `down` row groups below each other in turn, `rows` rows each.  The biases of its
// diagonals are looked up once, into LDS; a thread goes down its rows in steps of N, in which its vector slides over 2 N - 1 diagonals: N new
// ones a step, N stores of 16 bytes.

constexpr int kTileDiagonals = 4096;
template <int DT> struct VectorOf { static constexpr int value = DT == DDP_FP32 ? 4 : 8; };

template <int TT, int OT, bool ADD>
__global__ __launch_bounds__(kThreads) void apply_kernel(BiasArgs a) {
    constexpr int N = VectorOf<OT>::value;
    __shared__ __attribute__((aligned(16))) float of[kTileDiagonals];
    __shared__ int32_t first[kMaxBuckets];
    __shared__ float value[kMaxBuckets];             // of the head's buckets
    for (int k = threadIdx.x; k < a.sides; k += kThreads) first[k] = a.first[k];
    const int x = threadIdx.x & (a.cols - 1), y = threadIdx.x >> a.log2_cols;
    const int high = (kThreads >> a.log2_cols) * a.rows, wide = a.cols * N;
    for (int64_t turn = blockIdx.x; turn < a.tiles; turn += gridDim.x) {
        const int64_t tile = !ADD && a.regions ? tile_of_xcd(turn, a.tiles) : turn;
        const int64_t in_plane = tile % a.plane_tiles, plane = tile / a.plane_tiles, h = plane % a.heads, b = plane / a.heads;
        const int64_t c0 = in_plane % a.col_tiles * wide, i0 = in_plane / a.col_tiles * high;
        const int rows_here = static_cast<int>(min(a.queries - i0, int64_t(high))), cols_here = static_cast<int>(min(a.keys - c0, int64_t(wide)));
        // of[d]: of the diagonal that ends in the tile's first column d - high + 1 rows from its first row
        const int64_t r0 = c0 - i0 - (high - 1) - a.offset;
        __syncthreads();
        for (int k = threadIdx.x; k < a.buckets; k += kThreads)
            value[k] = load_one<TT>(a.table + (k * a.table_stride + h) * ElemBytes<TT>::value) * a.scale;
        __syncthreads();
        for (int d = high - rows_here + threadIdx.x; d < high - 1 + cols_here; d += kThreads) {
            const int64_t r = r0 + d;
            of[d] = !ADD && a.causal && r > 0 ? a.masked : value[bucket_of(first, a, r)];
        }
        __syncthreads();
        const int64_t c = c0 + x * N;
        if (c >= a.keys) continue;
        const int have = static_cast<int>(min(a.keys - c, int64_t(N)));
        const int seen = static_cast<int>(max(min(length_of(a.key_lengths, b, a.keys) - c, int64_t(N)), int64_t(0)));      // of the vector's keys
        const int64_t i_first = i0 + y * a.rows, i_end = min(i_first + a.rows, a.queries);
        const int at = x * N - y * a.rows + high - 1;                // of element 0 in the thread's first row
        char* out = a.scores + (b * a.s_batch + h * a.s_head + i_first * a.s_query + c) * ElemBytes<OT>::value;
        for (int g = 0; i_first + g < i_end; g += N) {
            const int rows = static_cast<int>(min(i_end - i_first - g, int64_t(N)));
            float window[2 * N - 1];                                 // of element e in row k: e - k + N - 1
#pragma unroll
            for (int k = 0; k < 2 * N - 1; ++k) window[k] = of[at - g - (N - 1) + k];
            // causal: element e of row k is visible where e - k <= edge
            const int64_t behind = i_first + g + a.offset - c;
            const int edge = a.causal ? static_cast<int>(max(min(behind, int64_t(N)), int64_t(-N))) : N;
            Parts<OT, N> there[N] = {};                              // all on the way together
            const bool some = seen > 0 && edge > -N;                 // (what is masked is not read)
            if constexpr (ADD) {
                if (have == N && some) {
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (k < rows) there[k] = load_parts<OT, N>(out + static_cast<int64_t>(g + k) * a.s_query * ElemBytes<OT>::value);
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k >= rows) break;
                char* to = out + static_cast<int64_t>(g + k) * a.s_query * ElemBytes<OT>::value;
                float v[N];
                if constexpr (ADD) {
                    if (have == N) widen<OT, N>(there[k], v);
                    else load_some<OT, N>(to, some ? have : 0, v);
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if constexpr (ADD) v[e] = e < seen && e - k <= edge ? window[e - k + N - 1] + v[e] : a.masked;
                    else v[e] = e < seen ? window[e - k + N - 1] : a.masked;
                }
                store_some<OT, N>(to, have, v);
            }
        }
    }
}

// ---- gradient ----
//
// (An element at a time with its bucket's sum in LDS took 1411 us of 2 x 16 x 4096 x 4096 where this takes 98.)
// A vector of N keys (16 bytes) that moves one vector to the right with every N rows meets the same 2 N - 1 diagonals in every such step:
// a lane holds them in registers, loads whole aligned vectors, and adds every element once.  Lane t of the band has columns N (g + t) in the
// rows N g ... N g + N - 1; neighbours in a wave are neighbours in memory.
//
// A block has the 64 lanes' band (64 N diagonals) of one head and a share of its row groups of all sequences, in equal parts for its waves.  Every
// kRun row groups, at most 64 N additions of a diagonal in binary32, the waves' diagonals are put together in LDS, and buckets, which are ranges of
// diagonals, summed in binary64 (one chain over 134 sequences of 4096 equal scores was off by 2^-9).
// Where no wave has more than that, the kernel goes without the loop over runs, whose scalars cost some 0.5 us (25 sequences of 97 queries and 15 keys
// 8.6 us, with it 9.2).
constexpr int64_t kRun = 64;

template <int N> struct Band {
    static constexpr int diagonals = 64 * N + N - 1, low = N - 1;    // element e of row x of lane t: N t + e - x + low
};
struct JoinArgs {
    const float* partial;
    char* grad;
    int64_t grad_stride;
    int32_t parts, heads, buckets, type, add;
    float scale;
};
// The diagonals that belong to bucket k, as r from lo to hi (hi < lo: none).
__device__ __forceinline__ void range_of(const int32_t* first, const BiasArgs& a, int k, int64_t& lo, int64_t& hi) {
    const bool behind = k >= a.sides;
    const int side = behind ? k - a.sides : k;
    const int64_t from = first[side], to = side + 1 < a.sides ? first[side + 1] - 1 : kFar;
    lo = behind ? (from > 1 ? from : 1) : -to;
    hi = behind ? to : side == 0 && !a.both ? kFar : -from;
}

// Strips of the longest diagonals come first, so that the short ones fill in at the end: from `center` to both sides, then what is left of one.
__device__ __forceinline__ int64_t strip_of(const BiasArgs& a, int64_t turn) {
    const int64_t below = a.center, above = a.strips - 1 - a.center, both = below < above ? below : above;
    if (turn <= 2 * both) return a.center + ((turn & 1) ? (turn + 1) / 2 : -(turn / 2));
    return below < above ? turn : a.strips - 1 - turn;
}

// A vector's elements from byte `by` on (0 to 15), then anything.
template <typename P>
__device__ __forceinline__ void shift_down(P& v, int by) {
    uint32_t* w = v.part[0].w;
    if (by & 8) {
        w[0] = w[2];
        w[1] = w[3];
    }
    if (by & 4) {
        w[0] = w[1];
        w[1] = w[2];
        w[2] = w[3];
    }
    if (by & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = w[i] >> 16 | (i < 3 ? w[i + 1] << 16 : 0u);
    }
}

template <int ST, bool NT, bool RUNS>
__global__ __launch_bounds__(kThreads) void diagonal_kernel(BiasArgs a, JoinArgs j) {
    constexpr int N = ST == DDP_FP32 ? 4 : 8, DIAGONALS = Band<N>::diagonals;
    __shared__ float diagonal[kWaves][DIAGONALS + 1];
    __shared__ int32_t first[kMaxBuckets];
    extern __shared__ double sums[];                 // of the buckets
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    for (int k = threadIdx.x; k < a.sides; k += kThreads) first[k] = a.first[k];
    for (int k = threadIdx.x; k < a.buckets; k += kThreads) sums[k] = 0.0;
    const int64_t h = blockIdx.x % a.heads;
    const int part = blockIdx.x / a.heads, share = part % a.shares;
    const int64_t groups = (a.queries + N - 1) / N, vectors = (a.keys + N - 1) / N;
    const char* scores = a.scores + h * a.s_head * ElemBytes<ST>::value;
    for (int64_t turn = part / a.shares; turn < a.strips; turn += a.strip_blocks) {
        const int64_t t0 = a.band0 + strip_of(a, turn) * 64;
        // the row groups in which some lane has a column, of all sequences, in equal parts for all waves of the shares
        const int64_t g_from = max(int64_t(0), -min(t0 + 63, a.last)), steps = max(min(groups, vectors - t0) - g_from, int64_t(0));
        const int64_t units = steps * a.batch, turns = static_cast<int64_t>(a.shares) * kWaves;
        const int64_t each = (units + turns - 1) / turns, mine = (static_cast<int64_t>(share) * kWaves + wave) * each;
        int64_t rest = min(each, units - mine), b = rest > 0 ? mine / steps : 0, g = g_from + (rest > 0 ? mine % steps : 0);
        for (int64_t runs = RUNS ? (each + kRun - 1) / kRun : 1; runs > 0; --runs) {
            float acc[2 * N - 1] = {};
            int64_t left = RUNS ? min(rest, kRun) : rest;
            rest -= left;
            while (left > 0) {
                const int64_t keys = length_of(a.key_lengths, b, a.keys), queries = length_of(a.query_lengths, b, a.queries);
                const int64_t here = min(left, g_from + steps - g), stop = g + here, end = min(stop, (queries + N - 1) / N);
                left -= here;
                const char* s = scores + b * a.s_batch * ElemBytes<ST>::value;
                const int64_t before = b * a.s_batch + h * a.s_head;         // of the scores' memory; room: from here to its end
                const int64_t room = (a.batch - 1 - b) * a.s_batch + (a.heads - 1 - h) * a.s_head + (a.queries - 1) * a.s_query + a.keys;
                for (; g < end; ++g) {
                    const int64_t i = g * N;
                    const int c = static_cast<int>(g + t0 + lane) * N;
                    const unsigned at = static_cast<unsigned>(c) * ElemBytes<ST>::value;
                    if (c < 0 || c >= keys || lane > a.last - t0) continue;
                    // (what follows a row's keys is read with them, as far as the tensor reaches, and not used)
                    if ((i + N - 1) * a.s_query + c + N <= room) {
                        Parts<ST, N> v[N];
#pragma unroll
                        for (int x = 0; x < N; ++x) v[x] = load_parts<ST, N, NT>(s + (i + x) * a.s_query * ElemBytes<ST>::value + at);
                        const bool partial = c + N > keys || i + N > queries;
                        const int have = static_cast<int>(min(keys - c, int64_t(N))), rows = static_cast<int>(min(queries - i, int64_t(N)));
                        if (__ballot(partial) != 0) {
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                const int in = have * ElemBytes<ST>::value - 4 * w;          // bytes of this word
                                const uint32_t keep = in >= 4 ? ~0u : in == 2 ? 0xFFFFu : 0u;
#pragma unroll
                                for (int x = 0; x < N; ++x) v[x].part[0].w[w] &= x < rows ? keep : 0u;
                            }
                        }
#pragma unroll
                        for (int x = 0; x < N; ++x) {
                            float e[N];
                            widen<ST, N>(v[x], e);
#pragma unroll
                            for (int k = 0; k < N; ++k) acc[k - x + N - 1] += e[k];
                        }
                    } else {
                        // in the tensor's last rows a vector that would reach over its end is moved back to end with it, and its elements down
                        // again; the sums go round instead of the rows being unrolled
                        const int have = static_cast<int>(min(keys - c, int64_t(N)));
                        const bool whole = before + room >= N;
                        auto place = [&](int x) { return (i + x) * a.s_query + c; };
                        auto row = [&](int x) { return load_parts<ST, N>(s + min(place(x), room - N) * ElemBytes<ST>::value); };
                        Parts<ST, N> next = {};
                        if (whole) next = row(0);
#pragma unroll 1
                        for (int x = 0; x < 2 * N - 1; ++x) {
                            if (x < N) {
                                Parts<ST, N> v = next;
                                float e[N];
                                if (whole) {
                                    next = row(min(x + 1, N - 1));
                                    shift_down(v, static_cast<int>(max(min(place(x) - room + N, int64_t(N - 1)), int64_t(0))) * ElemBytes<ST>::value);
                                    widen<ST, N>(v, e);
                                } else {
                                    load_some<ST, N>(s + (i + x) * a.s_query * ElemBytes<ST>::value + at, i + x < queries ? have : 0, e);
                                }
#pragma unroll
                                for (int k = 0; k < N; ++k) acc[k + N - 1] += k < have && i + x < queries ? e[k] : 0.0f;
                            }
                            const float last = acc[2 * N - 2];
#pragma unroll
                            for (int k = 2 * N - 2; k > 0; --k) acc[k] = acc[k - 1];
                            acc[0] = last;
                        }
                    }
                }
                g = stop;
                if (g == g_from + steps) {
                    ++b;
                    g = g_from;
                }
            }
            // diagonals of two neighbouring lanes: first each lane's upper ones (and the lowest lane's lower ones), then the others'
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) diagonal[wave][N * lane + k + N - 1] = acc[k + N - 1];
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < N - 1; ++k) diagonal[wave][k] = acc[k];
            }
            __syncthreads();
            if (lane > 0) {
#pragma unroll
                for (int k = 0; k < N - 1; ++k) diagonal[wave][N * lane + k] += acc[k];
            }
            __syncthreads();
            for (int d = threadIdx.x; d < DIAGONALS; d += kThreads) {
                float sum = diagonal[0][d];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) sum += diagonal[w][d];
                diagonal[0][d] = sum;
            }
            __syncthreads();
            // buckets go round the threads; those of many diagonals take a wave each
            const int64_t r0 = t0 * N - Band<N>::low - a.offset;         // of diagonal[0][0]
            const int64_t top = a.causal ? min(int64_t(0), r0 + DIAGONALS - 1) : r0 + DIAGONALS - 1;
            for (int k0 = wave * 64; k0 < a.buckets; k0 += kThreads) {
                int64_t lo = 0, hi = -1;
                if (k0 + lane < a.buckets) range_of(first, a, k0 + lane, lo, hi);
                const int d0 = static_cast<int>(max(lo, r0) - r0), n = static_cast<int>(max(min(hi, top) - max(lo, r0) + 1, int64_t(0)));
                if (n > 0 && n <= 16) {
                    double sum = 0.0;
                    for (int d = 0; d < n; ++d) sum += diagonal[0][d0 + d];
                    sums[k0 + lane] += sum;
                }
                for (uint64_t many = __ballot(n > 16); many != 0; many &= many - 1) {
                    const int l = __ffsll(static_cast<unsigned long long>(many)) - 1, from = __shfl(d0, l), count = __shfl(n, l);
                    double sum = 0.0;
                    for (int d = lane; d < count; d += 64) sum += diagonal[0][from + d];
#pragma unroll
                    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
                    if (lane == l) sums[k0 + l] += sum;
                }
            }
        }
    }
    __syncthreads();
    if (j.parts == 1) {                              // a head's sums are whole: no join (294 queries, 4 keys 10.6 -> 8.2 us)
        for (int k = threadIdx.x; k < a.buckets; k += kThreads) put_grad(j.grad, j.type, k * j.grad_stride + h, j.add, sums[k] * j.scale);
        return;
    }
    for (int k = threadIdx.x; k < a.buckets; k += kThreads) a.partial[(static_cast<int64_t>(part) * a.heads + h) * a.buckets + k] = static_cast<float>(sums[k]);
}

// A wave has 64 sums of a share of the parts, kJoinWaves of them meet in LDS.
constexpr int kJoinWaves = 16, kJoinDeep = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(JoinArgs a) {
    __shared__ double meet[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x * 64 + lane, all = a.heads * a.buckets;
    double sum = 0.0;
    if (at < all) {
        for (int p = wave; p < a.parts; p += kJoinWaves * kJoinDeep) {
            float x[kJoinDeep];                      // (no condition on a load: it would be waited for before the next)
#pragma unroll
            for (int u = 0; u < kJoinDeep; ++u) x[u] = a.partial[static_cast<int64_t>(min(p + u * kJoinWaves, a.parts - 1)) * all + at];
#pragma unroll
            for (int u = 0; u < kJoinDeep; ++u) sum += p + u * kJoinWaves < a.parts ? x[u] : 0.0f;
        }
    }
    meet[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || at >= all) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) sum += meet[w][lane];
    sum *= a.scale;
    const int h = at / a.buckets, k = at % a.buckets;
    put_grad(a.grad, a.type, k * a.grad_stride + h, a.add, sum);
}

// ---- host ----

constexpr int64_t kMaxTiles = int64_t(1) << 20, kTiles = 8192;
constexpr int kTileRows = 16;
// Blocks as many as are resident at once (1280 to 5120: within 3 %).  Scores of kStreamBytes and more, that no cache holds, are read past them
// (2 x 16 x 4096 x 4096 98 us against 104.5; 8 x 16 x 512 x 512 the other way 21.5 against 23.3).
constexpr int64_t kGradBlocks = 1792, kGradSteps = 4, kComputeUnits = 256, kStreamBytes = int64_t(1) << 28;
constexpr int64_t kPartBytes = int64_t(1) << 24;     // of the workspace, if 64 parts do not take more

template <int TT, int OT>
hipError_t launch_apply(ddp_position_bias* h, BiasArgs a, bool add) {
    constexpr int N = VectorOf<OT>::value;
    const int64_t vectors = (a.keys + N - 1) / N, planes = a.batch * a.heads;
    while (a.log2_cols < 8 && (1 << a.log2_cols) < vectors) ++a.log2_cols;
    a.cols = 1 << a.log2_cols;
    const int down = kThreads >> a.log2_cols;
    a.col_tiles = (vectors + a.cols - 1) / a.cols;
    // N rows a thread; where scores are added to, up to kTileRows, as many as leave kTiles tiles and fit the table (16 x 4096 x 4096 bfloat16, a few
    // calls: a fill 89 us with 8 rows and 101 with 16, added 171 and 165; added to 8 x 16 x 512 x 512 in binary32, 2048 tiles at least 57 us, 8192 48)
    a.rows = N;
    while (add && a.rows < kTileRows && (2 * a.rows * down + a.cols * N <= kTileDiagonals) && a.rows * down < a.queries &&
           planes * a.col_tiles * ((a.queries + 2 * a.rows * down - 1) / (2 * a.rows * down)) >= kTiles)
        a.rows *= 2;
    const int64_t high = static_cast<int64_t>(a.rows) * down;
    a.plane_tiles = a.col_tiles * ((a.queries + high - 1) / high);
    a.tiles = planes * a.plane_tiles;
    // A fill that no cache holds goes to a stretch of memory for each XCD (16 x 4096 x 4096 bfloat16 91 us, neighbouring tiles in different XCDs
    // 100; in rows that are three elements further apart 110 and 128; 16 x 2048 x 2048 28 and 26); what is read too does not (165 us, that way 186).
    a.regions = planes * a.queries * a.keys * ElemBytes<OT>::value >= kStreamBytes;
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(a.tiles, kMaxTiles));
    if (add) hipLaunchKernelGGL((apply_kernel<TT, OT, true>), dim3(blocks), dim3(kThreads), 0, h->stream, a);
    else hipLaunchKernelGGL((apply_kernel<TT, OT, false>), dim3(blocks), dim3(kThreads), 0, h->stream, a);
    return hipGetLastError();
}
template <int TT>
hipError_t launch_apply(ddp_position_bias* h, const BiasArgs& a, int out, bool add) {
    if (out == DDP_FP32) return launch_apply<TT, DDP_FP32>(h, a, add);
    if (out == DDP_FP16) return launch_apply<TT, DDP_FP16>(h, a, add);
    return launch_apply<TT, DDP_BF16>(h, a, add);
}

bool out_of_reach(int64_t n, int64_t stride) { return n > 1 && stride > (int64_t(1) << 46) / (n - 1); }

int32_t check_shape(ddp_position_bias* h, int64_t batch, int64_t queries, int64_t keys, int64_t offset, int32_t dtype, int32_t table_dtype,
                    int64_t table_stride) {
    if (batch < 0 || queries < 0 || keys < 0) return layer_fail(h, DDP_ERR_ARG, "position bias: batch, queries and keys are at least 0");
    if (batch > kMaxBatch || queries > kMaxLength || keys > kMaxLength || offset > kMaxLength || offset < -kMaxLength)
        return layer_fail(h, DDP_ERR_UNSUPPORTED, "position bias: more than 2^20 sequences, 2^24 queries or keys, or an offset beyond them");
    if (!known_dtype(dtype) || !known_dtype(table_dtype)) return layer_fail(h, DDP_ERR_ARG, "position bias: unknown dtype");
    if (table_stride < h->heads || table_stride > INT32_MAX) return layer_fail(h, DDP_ERR_ARG, "position bias: the table's stride is below the number of heads (or above 2^31 - 1)");
    return DDP_OK;
}

}  // namespace

extern "C" {

const char* ddp_position_bias_last_error(const ddp_position_bias* h) { return h ? h->err.c_str() : ddp_last_error(nullptr); }

int32_t ddp_position_bias_create(ddp_position_bias** out, int32_t device, void* stream, int32_t heads, int32_t buckets, int32_t exact,
                                 int64_t max_distance, int32_t both) {
    if (!out) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_position_bias_create: out is null");
    *out = nullptr;
    const int32_t status = layer_device("ddp_position_bias_create: bad device", device);
    if (status != DDP_OK) return status;
    if (heads < 1 || buckets < 1) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_position_bias_create: heads and buckets are at least 1");
    if (heads > kMaxHeads || buckets > kMaxBuckets || max_distance > kMaxDistance)
        return layer_fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_position_bias_create: more than 4096 heads, 1024 buckets or a distance of 2^20");
    if (both && buckets % 2) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_position_bias_create: an odd number of buckets for two directions");
    const int32_t sides = both ? buckets / 2 : buckets;
    if (exact < 1 || exact > sides) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_position_bias_create: exact is from 1 to the buckets of a direction");
    if (exact < sides && max_distance <= exact) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_position_bias_create: max_distance is above exact");
    ddp_position_bias* h = new (std::nothrow) ddp_position_bias();
    if (!h) return layer_fail(nullptr, DDP_ERR_HIP, "out of host memory");
    h->device = device;
    h->stream = static_cast<hipStream_t>(stream);
    h->heads = heads;
    h->buckets = buckets;
    h->exact = exact;
    h->both = both != 0;
    h->sides = sides;
    h->distance = max_distance;
    try {
        for (int k = 0; k < sides; ++k) h->first_host.push_back(k < exact ? k : first_distance(exact, max_distance, k - exact, sides - exact));
    } catch (...) {
        delete h;
        return layer_fail(nullptr, DDP_ERR_HIP, "out of host memory");
    }
    if (device != DDP_DEVICE_NONE) {
        const int64_t each = static_cast<int64_t>(heads) * buckets * 4;
        h->parts = static_cast<int32_t>(std::max<int64_t>(64, std::min<int64_t>(4096, kPartBytes / each)));
        const int64_t firsts = round_up(sides * 4, 256);
        hipError_t err = layer_alloc(h, firsts + h->parts * each);
        if (err == hipSuccess) {
            OnDevice on(device);
            err = taken(hipMemcpy(h->mem, h->first_host.data(), static_cast<size_t>(sides) * 4, hipMemcpyHostToDevice));
            if (err != hipSuccess) (void)taken(hipFree(h->mem));
        }
        if (err != hipSuccess) {
            delete h;
            return layer_fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        h->first = reinterpret_cast<int32_t*>(h->mem);
        h->partial = reinterpret_cast<float*>(h->mem + firsts);
    }
    *out = h;
    return DDP_OK;
}

int32_t ddp_position_bias_destroy(ddp_position_bias* h) {
    if (!h) return DDP_ERR_ARG;
    layer_release(h);
    delete h;
    return DDP_OK;
}

int32_t ddp_position_bias_buckets(const ddp_position_bias* h, int32_t* first) {
    if (!h) return DDP_ERR_ARG;
    if (!first) return DDP_ERR_ARG;
    std::copy(h->first_host.begin(), h->first_host.end(), first);
    return h->sides;
}

int32_t ddp_position_bias_apply(ddp_position_bias* h, int64_t batch, int64_t queries, int64_t keys, int64_t offset, const void* table,
                                int32_t table_dtype, int64_t table_stride, float scale, const int32_t* key_lengths, int32_t causal, float masked,
                                int32_t accumulate, void* out, int32_t out_dtype, int64_t batch_stride, int64_t head_stride, int64_t query_stride) {
    if (!h) return DDP_ERR_ARG;
    const int32_t status = check_shape(h, batch, queries, keys, offset, out_dtype, table_dtype, table_stride);
    if (status != DDP_OK) return status;
    const bool some = batch > 0 && queries > 0 && keys > 0;
    if (some) {
        // every place is written once: the three strides in the order of their size step over what the shorter ones span
        struct { int64_t n, stride; } d[3] = {{batch, batch_stride}, {h->heads, head_stride}, {queries, query_stride}};
        std::sort(d, d + 3, [](const auto& x, const auto& y) { return x.stride < y.stride; });
        int64_t span = keys;
        for (const auto& x : d) {
            if (x.n == 1) continue;
            if (x.stride < span) return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_apply: rows of the scores overlap");
            if (out_of_reach(x.n, x.stride)) return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_apply: scores of more than 2^46 elements");
            span += (x.n - 1) * x.stride;
        }
    }
    if (some && (!table || !out)) return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_apply: null pointer");
    if (misaligned(table, elem_bytes(table_dtype)) || misaligned(out, elem_bytes(out_dtype)) || misaligned(key_lengths, 4))
        return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_apply: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_position_bias_apply without a device");
    if (!some) return DDP_OK;
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    BiasArgs a{};
    a.first = h->first;
    a.key_lengths = key_lengths;
    a.table = static_cast<const char*>(table);
    a.scores = static_cast<char*>(out);
    a.batch = batch;
    a.queries = queries;
    a.keys = keys;
    a.offset = offset;
    a.table_stride = table_stride;
    a.s_batch = batch > 1 ? batch_stride : 0;        // (of one, the stride may be anything)
    a.s_head = h->heads > 1 ? head_stride : 0;
    a.s_query = queries > 1 ? query_stride : 0;
    a.heads = h->heads;
    a.buckets = h->buckets;
    a.sides = h->sides;
    a.both = h->both;
    a.causal = causal != 0;
    a.scale = scale;
    a.masked = masked;
    LAYER_HIP(h, table_dtype == DDP_FP32   ? launch_apply<DDP_FP32>(h, a, out_dtype, accumulate != 0)
                 : table_dtype == DDP_FP16 ? launch_apply<DDP_FP16>(h, a, out_dtype, accumulate != 0)
                                           : launch_apply<DDP_BF16>(h, a, out_dtype, accumulate != 0));
    return DDP_OK;
}

int32_t ddp_position_bias_grad(ddp_position_bias* h, int64_t batch, int64_t queries, int64_t keys, int64_t offset, const void* dscores, int32_t dtype,
                               int64_t batch_stride, int64_t head_stride, int64_t query_stride, float scale, const int32_t* key_lengths,
                               const int32_t* query_lengths, int32_t causal, int32_t accumulate, void* grad, int32_t grad_dtype, int64_t grad_stride) {
    if (!h) return DDP_ERR_ARG;
    const int32_t status = check_shape(h, batch, queries, keys, offset, dtype, grad_dtype, grad_stride);
    if (status != DDP_OK) return status;
    if (batch_stride < 0 || head_stride < 0 || query_stride < 0) return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_grad: a stride is below 0");
    if (out_of_reach(batch, batch_stride) || out_of_reach(h->heads, head_stride) || out_of_reach(queries, query_stride))
        return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_grad: scores of more than 2^46 elements");
    const bool some = batch > 0 && queries > 0 && keys > 0;
    if (!grad || (some && !dscores)) return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_grad: null pointer");
    if (misaligned(dscores, elem_bytes(dtype)) || misaligned(grad, elem_bytes(grad_dtype)) || misaligned(key_lengths, 4) || misaligned(query_lengths, 4))
        return layer_fail(h, DDP_ERR_ARG, "ddp_position_bias_grad: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_position_bias_grad without a device");
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    JoinArgs j{h->partial, static_cast<char*>(grad), grad_stride, 0, h->heads, h->buckets, grad_dtype, accumulate != 0, scale};
    if (some) {
        BiasArgs a{};
        a.first = h->first;
        a.key_lengths = key_lengths;
        a.query_lengths = query_lengths;
        a.scores = static_cast<char*>(const_cast<void*>(dscores));
        a.partial = h->partial;
        a.batch = batch;
        a.queries = queries;
        a.keys = keys;
        a.offset = offset;
        a.s_batch = batch > 1 ? batch_stride : 0;    // (of one, the stride may be anything)
        a.s_head = h->heads > 1 ? head_stride : 0;
        a.s_query = queries > 1 ? query_stride : 0;
        a.heads = h->heads;
        a.buckets = h->buckets;
        a.sides = h->sides;
        a.both = h->both;
        a.causal = causal != 0;
        // lanes of the band: from the one that ends with the last query's first key to the one of the first query's last key, without those
        // that are all behind the query
        const int64_t n = dtype == DDP_FP32 ? 4 : 8, groups = (queries + n - 1) / n;
        int64_t last = (keys + n - 1) / n - 1;
        if (causal) last = std::min(last, offset + n - 1 >= 0 ? (offset + n - 1) / n : -((-offset) / n));
        a.band0 = 1 - groups;
        a.last = last;
        a.strips = (last - a.band0 + 1 + 63) / 64;
        if (a.strips > 0) {
            a.center = std::max<int64_t>(0, std::min(a.strips - 1, (((keys + n - 1) / n - groups) / 2 - a.band0) / 64));
            a.strip_blocks = static_cast<int32_t>(std::min<int64_t>(a.strips, h->parts));
            const int64_t blocks = static_cast<int64_t>(a.strip_blocks) * h->heads, steps = batch * std::min(groups, last - a.band0 + 1);
            // kGradSteps row groups a wave, or fewer to have a block for each compute unit
            const int64_t shares = std::max(steps / (kWaves * kGradSteps), std::min(steps / kWaves, kComputeUnits / blocks));
            a.shares = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>({kGradBlocks / blocks, h->parts / a.strip_blocks, shares})));
            const int64_t parts = static_cast<int64_t>(a.strip_blocks) * a.shares;
            const dim3 grid(static_cast<unsigned>(parts * h->heads));
            j.parts = static_cast<int32_t>(parts);
            const size_t bytes = static_cast<size_t>(a.buckets) * 8;
            const bool stream = product_reaches(kStreamBytes, {batch, h->heads, queries, keys, elem_bytes(dtype)});
            const bool long_waves = batch * groups > kRun * kWaves * a.shares;           // (no strip has more row groups)
            auto launch = [&](auto st, auto nt, auto runs) {
                hipLaunchKernelGGL((diagonal_kernel<st.value, nt.value, runs.value>), grid, dim3(kThreads), bytes, h->stream, a, j);
            };
            auto typed = [&](auto nt, auto runs) {
                if (dtype == DDP_FP32) launch(std::integral_constant<int, DDP_FP32>(), nt, runs);
                else if (dtype == DDP_FP16) launch(std::integral_constant<int, DDP_FP16>(), nt, runs);
                else launch(std::integral_constant<int, DDP_BF16>(), nt, runs);
            };
            auto run = [&](auto nt) {
                if (long_waves) typed(nt, std::true_type());
                else typed(nt, std::false_type());
            };
            if (stream) run(std::true_type());
            else run(std::false_type());
        }
        LAYER_HIP(h, hipGetLastError());
    } else if (accumulate) {
        return DDP_OK;
    }
    if (j.parts == 1) return DDP_OK;
    hipLaunchKernelGGL(join_kernel, dim3(static_cast<unsigned>((h->heads * h->buckets + 63) / 64)), dim3(64 * kJoinWaves), 0, h->stream, j);
    LAYER_HIP(h, hipGetLastError());
    return DDP_OK;
}

}  // extern "C"
