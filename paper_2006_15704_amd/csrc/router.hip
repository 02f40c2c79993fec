// Routing of tokens to experts, its gradient, and the step of the balance bias.
//
//   s = softmax(logits) or sigmoid(logits),  key = s + bias
//   a group's score is the sum of its `top` largest keys; the experts of the `kept` best groups are open
//   the `chosen` largest open keys, descending, ties to the lower index;  w = scale s (/ the sum of the chosen s)
//   gradient: t = dw scale, renormalised (t - sum t w') / sum s;  softmax: s (t - sum t s),  sigmoid: t s (1 - s)
#include "layer_host.h"

struct ddp_router : ddp::LayerHandle {
    int32_t experts = 0, chosen = 0, groups = 0, kept = 0, top = 0, score = 0, renormalise = 0;
    float scale = 1.0f;
};

namespace {

using namespace ddp;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxExperts = 1024, kMaxChosen = 64, kMaxGroups = 64;
constexpr int64_t kMaxTokens = INT32_MAX;

struct RouteArgs {
    const char* logits;
    const float* bias;
    int32_t* experts_out;
    char* weights;
    int32_t* counts;
    int64_t tokens, stride;
    int32_t experts, chosen, groups, kept, top, score, renormalise, weights_type;
    int32_t log2_lanes, each, log2_group, listed;    // of a team: lanes, experts a lane, lanes a group, candidates
    int32_t room;                                    // keys (or a lane's sorted words) in LDS for each wave
    float scale;
};
struct RouteGradArgs {
    const char *logits, *dweights;
    const int32_t* experts_in;
    char* dlogits;
    int64_t tokens, stride, dstride;
    int32_t experts, chosen, score, renormalise, dweights_type, log2_lanes;
    float scale;
};

template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
// The largest key and the lowest index that has it.
__device__ __forceinline__ void wave_best(double& key, int& at) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const double k = __shfl_xor(key, d);
        const int i = __shfl_xor(at, d);
        if (k > key || (k == key && i < at)) {
            key = k;
            at = i;
        }
    }
}
__device__ __forceinline__ void store_weight(char* p, int type, int64_t at, float x) {
    if (type == DDP_FP32) store_one<DDP_FP32>(p + at * 4, x);
    else if (type == DDP_FP16) store_one<DDP_FP16>(p + at * 2, x);
    else store_one<DDP_BF16>(p + at * 2, x);
}
__device__ __forceinline__ float load_weight(const char* p, int type, int64_t at) {
    return type == DDP_FP32 ? load_one<DDP_FP32>(p + at * 4) : type == DDP_FP16 ? load_one<DDP_FP16>(p + at * 2) : load_one<DDP_BF16>(p + at * 2);
}
// What one lane of a wave has written to LDS another may read.
__device__ __forceinline__ void wave_meets() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr double kNone = -__builtin_huge_val();
constexpr float kMasked = -__builtin_huge_valf();

// ---- a token by a wave, in binary64 ----

// Score and key of an expert from its logit; `largest` and `sum` are the softmax's.
__device__ __forceinline__ double score64(int score, float x, float largest, double sum) {
    if (score == DDP_SCORE_SIGMOID) return 1.0 / (1.0 + exp(-static_cast<double>(x)));
    return x == kMasked ? 0.0 : exp(static_cast<double>(x) - largest) / sum;
}
__device__ __forceinline__ double key64(float x, double s, double bias) {
    const double key = s + bias;
    return x != kMasked && key > kNone ? key : kNone;            // (NaN is not above)
}

// keys: of the experts, in LDS.
template <int LT>
__device__ void route_token(const RouteArgs& a, int64_t t, double* keys, int32_t* counts) {
    const int lane = threadIdx.x & 63, per_group = a.experts / a.groups;
    const char* row = a.logits + t * a.stride * ElemBytes<LT>::value;
    auto logit = [&](int e) { return load_one<LT>(row + e * ElemBytes<LT>::value); };
    float largest = kMasked;
    double sum = 0.0;
    if (a.score == DDP_SCORE_SOFTMAX) {
        for (int e = lane; e < a.experts; e += 64) largest = fmaxf(largest, logit(e));
        largest = wave_max(largest);
        for (int e = lane; e < a.experts; e += 64) sum += logit(e) == kMasked ? 0.0 : exp(static_cast<double>(logit(e)) - largest);
        sum = wave_sum(sum);
    }
    for (int e = lane; e < a.experts; e += 64) keys[e] = key64(logit(e), score64(a.score, logit(e), largest, sum), a.bias != nullptr ? static_cast<double>(a.bias[e]) : 0.0);
    wave_meets();
    auto best = [&](auto open, double& k, int& at) {
        k = kNone;
        at = kMaxExperts;
        for (int e = lane; e < a.experts; e += 64)
            if (keys[e] > k && open(e)) {
                k = keys[e];
                at = e;
            }
        wave_best(k, at);
    };
    uint64_t open = ~uint64_t(0);
    if (a.kept < a.groups) {
        double rank = kNone;                         // lane g: of group g
        for (int g = 0; g < a.groups; ++g) {
            double total, k;
            int first, second;
            best([&](int e) { return e / per_group == g; }, total, first);
            if (a.top == 2) {
                best([&](int e) { return e / per_group == g && e != first; }, k, second);
                if (k > kNone) total += k;
            }
            if (lane == g) rank = total;
        }
        open = 0;
        for (int n = 0; n < a.kept; ++n) {
            double k = rank;
            int at = lane;
            wave_best(k, at);
            if (!(k > kNone)) break;
            open |= uint64_t(1) << at;
            if (lane == at) rank = kNone;
        }
    }
    double mine = 0.0, all = 0.0;                    // lane n: of the n-th choice
    int expert = -1;
    for (int n = 0; n < a.chosen; ++n) {
        double k;
        int at;
        best([&](int e) { return (open >> (e / per_group) & 1) != 0; }, k, at);
        if (!(k > kNone)) break;
        const double w = score64(a.score, logit(at), largest, sum);
        all += w;
        if (lane == n) {
            mine = w;
            expert = at;
        }
        wave_meets();
        if (lane == 0) keys[at] = kNone;
        wave_meets();
    }
    if (lane < a.chosen) {
        double w = mine * a.scale;
        if (a.renormalise) w = all > 0.0 ? w / all : 0.0;
        a.experts_out[t * a.chosen + lane] = expert;
        store_weight(a.weights, a.weights_type, t * a.chosen + lane, static_cast<float>(w));
        if (a.counts != nullptr && expert >= 0) atomicAdd(&counts[expert], 1);
    }
    wave_meets();
}

__device__ __forceinline__ void clear_counts(const RouteArgs& a, int32_t* counts) {
    if (a.counts == nullptr) return;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) counts[e] = 0;
    __syncthreads();
}
__device__ __forceinline__ void add_counts(const RouteArgs& a, const int32_t* counts) {
    if (a.counts == nullptr) return;
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kThreads)
        if (counts[e] != 0) atomicAdd(a.counts + e, counts[e]);
}

// Groups that no team's lanes divide into.
template <int LT>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    extern __shared__ double keys[];                 // [kWaves][experts], then the counts
    int32_t* counts = reinterpret_cast<int32_t*>(keys + kWaves * a.experts);
    clear_counts(a, counts);
    const int wave = threadIdx.x >> 6;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * kWaves)
        route_token<LT>(a, t, keys + wave * a.experts, counts);
    add_counts(a, counts);
}

// ---- a token by a team ----
//
// A team of 1 to 64 lanes has up to kEach neighbouring experts a lane.  Keys in binary32 become words that sort as they do, with the place
// in the lane for their last four bits; a lane sorts its own, and the team takes the largest head, as often as there are candidates: two more than
// are chosen.  Where the candidates' keys are all further apart than the error of a binary32 key, their order is that of binary64.
// Where not, the candidates alone (or the groups) are put in order in binary64.  And where that leaves open whether all that belong are among them, a wave
// does the token over: one token in some thousands of 16-bit logits, hardly any other.

constexpr int kEach = 16, kSpare = 2;
// A key's error in parts of 2^-24 of the largest score and bias: exp, sum and quotient of a softmax over 1024 under 30, the key's
// rounding 1, the bits given to the place 32: two keys 126.
constexpr float kApart = 0x1p-16f;

template <int CTRL>
__device__ __forceinline__ uint32_t lane_moved(uint32_t x) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, true));
}
// x and what the neighbour group's lane has, step by step until all 2^log2 lanes have met.
template <typename F>
__device__ __forceinline__ void meet_lanes(int log2, F f) {
    if (log2 > 0) f([](uint32_t x) { return lane_moved<0xB1>(x); });         // quad_perm: 1 0 3 2
    if (log2 > 1) f([](uint32_t x) { return lane_moved<0x4E>(x); });         // quad_perm: 2 3 0 1
    if (log2 > 2) f([](uint32_t x) { return lane_moved<0x141>(x); });        // row_half_mirror
    if (log2 > 3) f([](uint32_t x) { return lane_moved<0x140>(x); });        // row_mirror
    if (log2 > 4) f([](uint32_t x) { return static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), 16)); });
    if (log2 > 5) f([](uint32_t x) { return static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), 32)); });
}
__device__ __forceinline__ float as_float(uint32_t x) { return __builtin_bit_cast(float, x); }
__device__ __forceinline__ uint32_t as_bits(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float team_sum(int log2, float x) {
    meet_lanes(log2, [&](auto move) { x += as_float(move(as_bits(x))); });
    return x;
}
__device__ __forceinline__ float team_max(int log2, float x) {
    meet_lanes(log2, [&](auto move) { x = fmaxf(x, as_float(move(as_bits(x)))); });
    return x;
}
__device__ __forceinline__ uint32_t team_max(int log2, uint32_t x) {
    meet_lanes(log2, [&](auto move) { x = max(x, move(x)); });
    return x;
}

// Words that sort as the floats do; 0 is below all of them.
__device__ __forceinline__ uint32_t sortable(float x) {
    const uint32_t b = as_bits(x);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_of(uint32_t word) {
    const uint32_t w = word & ~15u;
    return as_float(w >> 31 ? w ^ 0x80000000u : ~w);
}

// Descending, by odd-even merges.
template <int N>
__device__ __forceinline__ void sort_words(uint32_t (&w)[N]) {
#pragma unroll
    for (int p = 1; p < N; p <<= 1)
#pragma unroll
        for (int k = p; k >= 1; k >>= 1)
#pragma unroll
            for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const uint32_t x = w[i + j], y = w[i + j + k];
                        w[i + j] = max(x, y);
                        w[i + j + k] = min(x, y);
                    }
}

__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// EACH: the lane's experts, a.each of them used.
template <int LT, int EACH>
__global__ __launch_bounds__(kThreads) void route_team_kernel(RouteArgs a) {
    extern __shared__ double keys[];                 // [kWaves][room], then candidates and counts
    const int lanes = 1 << a.log2_lanes, l = threadIdx.x & (lanes - 1), team = threadIdx.x >> a.log2_lanes, teams = kThreads >> a.log2_lanes;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    char* behind = reinterpret_cast<char*>(keys + kWaves * a.room);
    uint32_t* word = reinterpret_cast<uint32_t*>(behind) + team * a.listed;          // of each candidate: its key, then its weight
    int32_t* at = reinterpret_cast<int32_t*>(behind) + (teams + team) * a.listed;    // its expert, or -1
    int32_t* counts = reinterpret_cast<int32_t*>(behind) + 2 * teams * a.listed;
    uint32_t* sorted = reinterpret_cast<uint32_t*>(keys + wave * a.room) + lane;     // the lane's words, 64 apart
    clear_counts(a, counts);
    const int e0 = l * a.each, mine = max(min(a.experts - e0, a.each), 0);
    float bias[EACH], of_bias = 0.0f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        bias[i] = a.bias != nullptr && i < mine ? a.bias[e0 + i] : 0.0f;
        of_bias = fmaxf(of_bias, fabsf(bias[i]) < __builtin_huge_valf() ? fabsf(bias[i]) : 0.0f);
    }
    of_bias = team_max(a.log2_lanes, of_bias);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * teams; base < a.tokens; base += static_cast<int64_t>(gridDim.x) * teams) {
        const int64_t t = base + team;
        const bool live = t < a.tokens;
        const char* row = a.logits + t * a.stride * ElemBytes<LT>::value;
        float x[EACH];
        if constexpr (EACH * ElemBytes<LT>::value >= 16) {
            if (live && mine == EACH) {
                widen<LT, EACH>(load_parts<LT, EACH>(row + e0 * ElemBytes<LT>::value), x);
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i) x[i] = live && i < mine ? load_one<LT>(row + (e0 + i) * ElemBytes<LT>::value) : kMasked;
            }
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = live && i < mine ? load_one<LT>(row + (e0 + i) * ElemBytes<LT>::value) : kMasked;
        }
        float largest = 0.0f, sum = 0.0f, most = 1.0f, s[EACH];
        if (a.score == DDP_SCORE_SOFTMAX) {
            largest = x[0];
#pragma unroll
            for (int i = 1; i < EACH; ++i) largest = fmaxf(largest, x[i]);
            largest = team_max(a.log2_lanes, largest);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s[i] = x[i] == kMasked ? 0.0f : fast_exp(x[i] - largest);
                sum += s[i];
            }
            sum = team_sum(a.log2_lanes, sum);
            most = 1.0f / sum;
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] *= most;
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] = __builtin_amdgcn_rcpf(1.0f + fast_exp(-x[i]));
        }
        const float apart = kApart * (most + of_bias);
        uint32_t w[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float key = s[i] + bias[i];
            w[i] = x[i] != kMasked && key > kMasked ? (sortable(key) & ~15u) | static_cast<uint32_t>(15 - i) : 0u;
        }
        sort_words<EACH>(w);
        bool again = false;                          // the token is for a wave
        const int of_team0 = lane & ~(lanes - 1);
        double sum64 = 0.0;                          // of the softmax, where it is asked for
        auto take_sum64 = [&]() {
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum64 += x[i] == kMasked ? 0.0 : exp(static_cast<double>(x[i]) - largest);
            for (int d = 1; d < lanes; d <<= 1) sum64 += __shfl_xor(sum64, d);
        };
        if (a.kept < a.groups) {
            float first = w[0] != 0 ? key_of(w[0]) : kMasked, second = kMasked;
            if constexpr (EACH > 1) second = w[1] != 0 ? key_of(w[1]) : kMasked;
            meet_lanes(a.log2_group, [&](auto move) {
                const float f = as_float(move(as_bits(first))), g = as_float(move(as_bits(second)));
                second = fmaxf(fminf(first, f), fmaxf(second, g));
                first = fmaxf(first, f);
            });
            const float rank = a.top == 2 && second > kMasked ? first + second : first;
            const int group = l >> a.log2_group;
            int before = 0;
            for (int g = 0; g < a.groups; ++g) {
                const float r = __shfl(rank, of_team0 + (g << a.log2_group));
                before += r > rank || (r == rank && g < group);
            }
            const float worst = -team_max(a.log2_lanes, before < a.kept && group < a.groups ? -rank : kMasked);
            const float next = team_max(a.log2_lanes, before >= a.kept && group < a.groups ? rank : kMasked);
            const bool close = live && next > kMasked && !(worst - next > 2.0f * apart);
            if (__ballot(close) != 0) {
                if (a.score == DDP_SCORE_SOFTMAX) take_sum64();
                double first64 = kNone, second64 = kNone;
#pragma unroll 1
                for (int i = 0; i < EACH; ++i) {
                    float v = kMasked, of_v = 0.0f;
#pragma unroll
                    for (int j = 0; j < EACH; ++j)
                        if (j == i) {
                            v = x[j];
                            of_v = bias[j];
                        }
                    const double key = key64(v, score64(a.score, v, largest, sum64), static_cast<double>(of_v));
                    second64 = fmax(fmin(first64, key), second64);
                    first64 = fmax(first64, key);
                }
                for (int d = 1; d < 1 << a.log2_group; d <<= 1) {
                    const double f = __shfl_xor(first64, d), g = __shfl_xor(second64, d);
                    second64 = fmax(fmin(first64, f), fmax(second64, g));
                    first64 = fmax(first64, f);
                }
                const double rank64 = a.top == 2 && second64 > kNone ? first64 + second64 : first64;
                int before64 = 0;
                for (int g = 0; g < a.groups; ++g) {
                    const double r = __shfl(rank64, of_team0 + (g << a.log2_group));
                    before64 += r > rank64 || (r == rank64 && g < group);
                }
                if (close) before = before64;
            }
            if (before >= a.kept) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) w[i] = 0;
            }
        }
#pragma unroll
        for (int i = 1; i < EACH; ++i) sorted[i * 64] = w[i];
        float left = kMasked;                        // the largest key behind the candidates
        int taken = 0;
        for (int n = 0; n <= a.listed; ++n) {
            const uint32_t head = w[0] >> 4, top = team_max(a.log2_lanes, head);
            if (n == a.listed) {
                if (top != 0) left = key_of(top << 4);
                break;
            }
            const uint64_t same = __ballot(head == top) >> of_team0;
            if (__ffsll(static_cast<unsigned long long>(same)) - 1 == l) {
                word[n] = w[0];
                at[n] = top != 0 ? e0 + 15 - static_cast<int>(w[0] & 15u) : -1;
                ++taken;
                w[0] = taken < EACH ? sorted[taken * 64] : 0u;
            }
        }
        wave_meets();
        // candidates go round the lanes: are two of the first a.chosen + 1 too near each other?
        bool near = false;
        for (int n = l; n < a.chosen; n += lanes) {
            const uint32_t here = word[n], behind = n + 1 < a.listed ? word[n + 1] : 0u;
            if (here != 0 && (behind != 0 || n + 1 >= a.listed)) {
                const float k = key_of(here), b = n + 1 < a.listed ? key_of(behind) : left;
                near |= b > kMasked && !(k - b > apart);
            }
        }
        const uint64_t of_team = lanes == 64 ? ~uint64_t(0) : (uint64_t(1) << lanes) - 1;
        const bool close = (__ballot(near) >> of_team0 & of_team) != 0;
        bool order64 = false;
        if (__ballot(close && live) != 0) {
            order64 = close;
            if (a.score == DDP_SCORE_SOFTMAX && a.bias != nullptr && sum64 == 0.0) take_sum64();
            if (a.bias == nullptr) sum64 = 1.0;
            // the wave's room for keys holds the candidates'
            double* exact = keys + wave * a.room + (team & ((64 >> a.log2_lanes) - 1)) * a.listed;
            for (int n = l; n < a.listed; n += lanes) {
                const int e = at[n];
                const float v = e >= 0 && live ? load_one<LT>(row + e * ElemBytes<LT>::value) : kMasked;
                exact[n] = e >= 0 ? key64(v, score64(a.score, v, largest, sum64), a.bias != nullptr ? static_cast<double>(a.bias[e]) : 0.0) : kNone;
            }
            wave_meets();
            if (order64) {
                double last = __builtin_huge_val();  // the lowest key that is chosen
                for (int n = l; n < a.listed; n += lanes) {
                    int rank = n;
                    if (at[n] >= 0) {
                        rank = 0;
                        for (int m = 0; m < a.listed; ++m) rank += at[m] >= 0 && (exact[m] > exact[n] || (exact[m] == exact[n] && (at[m] & 0xFFFF) < (at[n] & 0xFFFF)));
                        if (rank < a.chosen) last = fmin(last, exact[n]);
                    }
                    word[n] = static_cast<uint32_t>(rank);
                }
                float scale64 = 1.0f;                // (keys of a softmax without a bias are not divided by its sum)
                if (a.score == DDP_SCORE_SOFTMAX && a.bias == nullptr) scale64 = most;
                again = left > kMasked && !(static_cast<float>(last * scale64) - left > apart);
            }
            // one lane of a team decides for all
            again = (__ballot(again) >> of_team0 & of_team) != 0;
        }
        wave_meets();
        if (live && !again) {
            float all = 0.0f;
            for (int n = l; n < a.listed; n += lanes) {
                const int rank = order64 ? static_cast<int>(word[n]) : n, e = at[n];
                float v = 0.0f;
                if (rank < a.chosen && e >= 0) {
                    const float logit = load_one<LT>(row + e * ElemBytes<LT>::value);
                    v = a.score == DDP_SCORE_SOFTMAX ? expf(logit - largest) * most : 1.0f / (1.0f + expf(-logit));
                }
                all += v;
                word[n] = as_bits(v);
                at[n] = rank < a.chosen ? (e < 0 ? -1 : e | rank << 16) : -2;
                if (rank < a.chosen && e < 0) {
                    a.experts_out[t * a.chosen + rank] = -1;
                    store_weight(a.weights, a.weights_type, t * a.chosen + rank, 0.0f);
                }
            }
            all = team_sum(a.log2_lanes, all);
            const float factor = !a.renormalise ? a.scale : all > 0.0f ? a.scale / all : 0.0f;
            for (int n = l; n < a.listed; n += lanes) {
                if (at[n] < 0) continue;
                const int e = at[n] & 0xFFFF, rank = at[n] >> 16;
                a.experts_out[t * a.chosen + rank] = e;
                store_weight(a.weights, a.weights_type, t * a.chosen + rank, as_float(word[n]) * factor);
                if (a.counts != nullptr) atomicAdd(&counts[e], 1);
            }
        }
        for (uint64_t left_over = __ballot(live && again && l == 0); left_over != 0; left_over &= left_over - 1) {
            const int which = __ffsll(static_cast<unsigned long long>(left_over)) - 1;
            wave_meets();
            route_token<LT>(a, base + ((static_cast<int>(threadIdx.x & ~63u) + which) >> a.log2_lanes), keys + wave * a.room, counts);
        }
        wave_meets();
    }
    add_counts(a, counts);
}

__global__ __launch_bounds__(kThreads) void clear_kernel(int32_t* counts, int n) {
    for (int e = threadIdx.x; e < n; e += kThreads) counts[e] = 0;
}

// A token's gradient by a team of lanes with EACH neighbouring experts each.  What the chosen experts get is put together in a row in LDS, which is zeros
// otherwise, and everyone reads what is theirs; of sigmoids nothing else is computed.
template <int LT, int EACH>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteGradArgs a) {
    extern __shared__ float lds[];                   // [teams]: the row, then of the chosen: gradient, score, expert
    const int lanes = 1 << a.log2_lanes, l = threadIdx.x & (lanes - 1), team = threadIdx.x >> a.log2_lanes, teams = kThreads >> a.log2_lanes;
    constexpr int STEP = EACH + 4;                   // (lanes four words further apart: fewer of them share a bank)
    float* row = lds + team * (lanes * STEP + 3 * a.chosen);
    float* of = row + lanes * STEP;
    float* score = of + a.chosen;
    int32_t* at = reinterpret_cast<int32_t*>(score + a.chosen);
    auto place = [](int e) { return e / EACH * STEP + e % EACH; };
#pragma unroll
    for (int i = 0; i < EACH; ++i) row[l * STEP + i] = 0.0f;
    const int e0 = l * EACH, mine = max(min(a.experts - e0, EACH), 0);
    const int of_team0 = static_cast<int>(threadIdx.x & 63) & ~(lanes - 1);
    const uint64_t of_team = lanes == 64 ? ~uint64_t(0) : (uint64_t(1) << lanes) - 1;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * teams; base < a.tokens; base += static_cast<int64_t>(gridDim.x) * teams) {
        const int64_t t = base + team;
        const bool live = t < a.tokens;
        const char* from = a.logits + t * a.stride * ElemBytes<LT>::value;
        float s[EACH], largest = 0.0f, part = 0.0f;
        if (a.score == DDP_SCORE_SOFTMAX) {
            load_some<LT, EACH>(from + e0 * ElemBytes<LT>::value, live ? mine : 0, s);
            largest = kMasked;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i < mine) largest = fmaxf(largest, s[i]);
            largest = team_max(a.log2_lanes, largest);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s[i] = i >= mine || s[i] == kMasked ? 0.0f : expf(s[i] - largest);
                part += s[i];
            }
            part = 1.0f / team_sum(a.log2_lanes, part);
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] *= part;
        }
        // the chosen go round the lanes
        bool any = false;
        float all = 0.0f, dot = 0.0f;
        for (int n = l; n < a.chosen; n += lanes) {
            const int e = live ? a.experts_in[t * a.chosen + n] : -1;
            const bool named = e >= 0 && e < a.experts;
            float w = 0.0f, g = 0.0f;
            if (named) {
                const float x = load_one<LT>(from + e * ElemBytes<LT>::value);
                w = a.score == DDP_SCORE_SIGMOID ? 1.0f / (1.0f + expf(-x)) : x == kMasked ? 0.0f : expf(x - largest) * part;
                g = load_weight(a.dweights, a.dweights_type, t * a.chosen + n) * a.scale;
            }
            any |= named;
            all += w;
            dot += g * w;
            at[n] = named ? e : -1;
            of[n] = g;
            score[n] = w;
        }
        any = (__ballot(any) >> of_team0 & of_team) != 0;
        if (a.renormalise) {
            all = team_sum(a.log2_lanes, all);
            dot = team_sum(a.log2_lanes, dot);
            const float mean = dot / all;
            dot = 0.0f;
            for (int n = l; n < a.chosen; n += lanes) {
                const float g = at[n] >= 0 && all > 0.0f ? (of[n] - mean) / all : 0.0f;
                of[n] = g;
                dot += g * score[n];
            }
        }
        dot = a.score == DDP_SCORE_SOFTMAX ? team_sum(a.log2_lanes, dot) : 0.0f;
        wave_meets();
        for (int n = l; n < a.chosen; n += lanes) {
            const int e = at[n];
            if (e < 0) continue;
            float sum = 0.0f;                        // (an expert that is named twice)
            for (int m = 0; m < a.chosen; ++m) sum += at[m] == e ? of[m] : 0.0f;
            if (a.score == DDP_SCORE_SIGMOID) {
                const float x = load_one<LT>(from + e * ElemBytes<LT>::value);
                sum *= score[n] * (1.0f / (1.0f + expf(x)));     // 1 - s, without the difference
            }
            row[place(e)] = sum;
        }
        wave_meets();
        float d[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            d[i] = row[l * STEP + i];
            if (a.score == DDP_SCORE_SOFTMAX) d[i] = any ? s[i] * (d[i] - dot) : 0.0f;
        }
        if (live && mine > 0) store_some<LT, EACH>(a.dlogits + (t * a.dstride + e0) * ElemBytes<LT>::value, mine, d);
        wave_meets();
        for (int n = l; n < a.chosen; n += lanes)
            if (at[n] >= 0) row[place(at[n])] = 0.0f;
    }
}

// A thread an expert; the mean is compared in whole numbers.
__global__ __launch_bounds__(kMaxExperts) void balance_kernel(const int32_t* counts, int replicas, int experts, float rate, const float* bias, float* out) {
    __shared__ int64_t part[kMaxExperts / 64];
    const int e = threadIdx.x;
    int64_t mine = 0;
    for (int r = 0; r < replicas; ++r) mine += e < experts ? counts[static_cast<int64_t>(r) * experts + e] : 0;
    const int64_t of_wave = wave_sum(mine);
    if ((e & 63) == 0) part[e >> 6] = of_wave;
    __syncthreads();
    int64_t all = 0;
    for (int w = 0; w < kMaxExperts / 64; ++w) all += part[w];
    if (e < experts) out[e] = bias[e] + (mine * experts < all ? rate : mine * experts > all ? -rate : 0.0f);
}

// ---- host ----

constexpr int64_t kBlocks = 2048;

// The team of a token: a.each experts a lane, the most that divide into its groups.  False: none.
bool find_team(RouteArgs& a) {
    const int per_group = a.experts / a.groups;
    if (a.kept >= a.groups) {
        a.each = std::min({kEach, (a.experts + 3) / 4, 256 / a.chosen + 4});     // (many candidates take more lanes: their LDS is a team's)
    } else {
        for (a.each = std::min(kEach, per_group); a.each > 0; --a.each) {
            const int lanes = per_group / a.each;
            if (per_group % a.each == 0 && (lanes & (lanes - 1)) == 0) break;
        }
        if (a.each == 0) return false;
        while (a.each << a.log2_group < per_group) ++a.log2_group;
    }
    while (a.each << a.log2_lanes < a.experts) ++a.log2_lanes;
    if (a.log2_lanes > 6) return false;
    a.listed = std::min(a.chosen + kSpare, a.experts);
    a.room = std::max({a.experts, (64 >> a.log2_lanes) * a.listed, 32 * (a.each > 8 ? 16 : a.each > 4 ? 8 : a.each > 2 ? 4 : a.each)});
    return true;
}
template <int LT>
hipError_t launch_route(ddp_router* h, RouteArgs a) {
    const size_t counts = static_cast<size_t>(a.experts) * 4;
    if (!find_team(a)) {
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, kBlocks));
        hipLaunchKernelGGL((route_kernel<LT>), dim3(blocks), dim3(kThreads), static_cast<size_t>(kWaves) * a.experts * 8 + counts, h->stream, a);
        return hipGetLastError();
    }
    const int teams = kThreads >> a.log2_lanes;
    const dim3 blocks(static_cast<unsigned>(std::min<int64_t>((a.tokens + teams - 1) / teams, kBlocks))), threads(kThreads);
    const size_t bytes = static_cast<size_t>(kWaves) * a.room * 8 + static_cast<size_t>(teams) * a.listed * 8 + counts;
    if (a.each > 8) hipLaunchKernelGGL((route_team_kernel<LT, 16>), blocks, threads, bytes, h->stream, a);
    else if (a.each > 4) hipLaunchKernelGGL((route_team_kernel<LT, 8>), blocks, threads, bytes, h->stream, a);
    else if (a.each > 2) hipLaunchKernelGGL((route_team_kernel<LT, 4>), blocks, threads, bytes, h->stream, a);
    else if (a.each > 1) hipLaunchKernelGGL((route_team_kernel<LT, 2>), blocks, threads, bytes, h->stream, a);
    else hipLaunchKernelGGL((route_team_kernel<LT, 1>), blocks, threads, bytes, h->stream, a);
    return hipGetLastError();
}
template <int LT>
hipError_t launch_grad(ddp_router* h, RouteGradArgs a) {
    const int each = a.experts > 256 || (a.experts > 32 && 4 * a.chosen <= a.experts) ? 16 : 4;      // (many chosen take more lanes: their LDS is a team's)
    while (each << a.log2_lanes < a.experts) ++a.log2_lanes;
    const int teams = kThreads >> a.log2_lanes;
    const dim3 blocks(static_cast<unsigned>(std::min<int64_t>((a.tokens + teams - 1) / teams, kBlocks))), threads(kThreads);
    const size_t bytes = static_cast<size_t>(teams) * (((each + 4) << a.log2_lanes) + 3 * a.chosen) * 4;
    if (each == 16) hipLaunchKernelGGL((route_grad_kernel<LT, 16>), blocks, threads, bytes, h->stream, a);
    else hipLaunchKernelGGL((route_grad_kernel<LT, 4>), blocks, threads, bytes, h->stream, a);
    return hipGetLastError();
}

int32_t check_tokens(ddp_router* h, int64_t tokens, int32_t dtype, int32_t weights_dtype, int64_t stride) {
    if (tokens < 0 || tokens > kMaxTokens) return layer_fail(h, DDP_ERR_ARG, "router: tokens outside [0, 2^31 - 1]");
    if (!known_dtype(dtype) || !known_dtype(weights_dtype)) return layer_fail(h, DDP_ERR_ARG, "router: unknown dtype");
    if (stride < h->experts || stride > INT32_MAX) return layer_fail(h, DDP_ERR_ARG, "router: a stride is below the number of experts (or above 2^31 - 1)");
    return DDP_OK;
}

}  // namespace

extern "C" {

const char* ddp_router_last_error(const ddp_router* h) { return h ? h->err.c_str() : ddp_last_error(nullptr); }

int32_t ddp_router_create(ddp_router** out, int32_t device, void* stream, int32_t experts, int32_t chosen, int32_t groups, int32_t kept, int32_t top,
                          int32_t score, int32_t renormalise, float scale) {
    if (!out) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: out is null");
    *out = nullptr;
    const int32_t status = layer_device("ddp_router_create: bad device", device);
    if (status != DDP_OK) return status;
    if (experts < 1 || chosen < 1 || groups < 1 || kept < 1) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: experts, chosen, groups and kept are at least 1");
    if (experts > kMaxExperts || chosen > kMaxChosen || groups > kMaxGroups)
        return layer_fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_router_create: more than 1024 experts, 64 chosen ones or 64 groups");
    if (experts % groups != 0 || kept > groups || chosen > experts / groups * kept)
        return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: groups are of equal size, and the kept ones hold the chosen experts");
    if (top != 1 && top != 2) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: a group's score is its largest key or the sum of two");
    if (score != DDP_SCORE_SOFTMAX && score != DDP_SCORE_SIGMOID) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: unknown score");
    if (!(scale - scale == 0.0f)) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_router_create: scale is not finite");
    ddp_router* h = new (std::nothrow) ddp_router();
    if (!h) return layer_fail(nullptr, DDP_ERR_HIP, "out of host memory");
    h->device = device;
    h->stream = static_cast<hipStream_t>(stream);
    h->experts = experts;
    h->chosen = chosen;
    h->groups = groups;
    h->kept = kept;
    h->top = top;
    h->score = score;
    h->renormalise = renormalise != 0;
    h->scale = scale;
    *out = h;
    return DDP_OK;
}

int32_t ddp_router_destroy(ddp_router* h) {
    if (!h) return DDP_ERR_ARG;
    layer_release(h);
    delete h;
    return DDP_OK;
}

int32_t ddp_router_route(ddp_router* h, int64_t tokens, const void* logits, int32_t dtype, int64_t stride, const float* bias, int32_t* experts_out,
                         void* weights, int32_t weights_dtype, int32_t* counts, int32_t accumulate) {
    if (!h) return DDP_ERR_ARG;
    const int32_t status = check_tokens(h, tokens, dtype, weights_dtype, stride);
    if (status != DDP_OK) return status;
    if (tokens > 0 && (!logits || !experts_out || !weights)) return layer_fail(h, DDP_ERR_ARG, "ddp_router_route: null pointer");
    if (misaligned(logits, elem_bytes(dtype)) || misaligned(bias, 4) || misaligned(experts_out, 4) || misaligned(weights, elem_bytes(weights_dtype)) ||
        misaligned(counts, 4))
        return layer_fail(h, DDP_ERR_ARG, "ddp_router_route: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_router_route without a device");
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    if (counts && !accumulate) {
        hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(kThreads), 0, h->stream, counts, h->experts);
        LAYER_HIP(h, hipGetLastError());
    }
    if (tokens == 0) return DDP_OK;
    RouteArgs a{};
    a.logits = static_cast<const char*>(logits);
    a.bias = bias;
    a.experts_out = experts_out;
    a.weights = static_cast<char*>(weights);
    a.counts = counts;
    a.tokens = tokens;
    a.stride = stride;
    a.experts = h->experts;
    a.chosen = h->chosen;
    a.groups = h->groups;
    a.kept = h->kept;
    a.top = h->top;
    a.score = h->score;
    a.renormalise = h->renormalise;
    a.weights_type = weights_dtype;
    a.scale = h->scale;
    LAYER_HIP(h, dtype == DDP_FP32 ? launch_route<DDP_FP32>(h, a) : dtype == DDP_FP16 ? launch_route<DDP_FP16>(h, a) : launch_route<DDP_BF16>(h, a));
    return DDP_OK;
}

int32_t ddp_router_grad(ddp_router* h, int64_t tokens, const void* logits, int32_t dtype, int64_t stride, const int32_t* experts_in,
                        const void* dweights, int32_t dweights_dtype, void* dlogits, int64_t dlogits_stride) {
    if (!h) return DDP_ERR_ARG;
    int32_t status = check_tokens(h, tokens, dtype, dweights_dtype, stride);
    if (status == DDP_OK) status = check_tokens(h, tokens, dtype, dweights_dtype, dlogits_stride);
    if (status != DDP_OK) return status;
    if (tokens > 0 && (!logits || !experts_in || !dweights || !dlogits)) return layer_fail(h, DDP_ERR_ARG, "ddp_router_grad: null pointer");
    if (misaligned(logits, elem_bytes(dtype)) || misaligned(experts_in, 4) || misaligned(dweights, elem_bytes(dweights_dtype)) ||
        misaligned(dlogits, elem_bytes(dtype)))
        return layer_fail(h, DDP_ERR_ARG, "ddp_router_grad: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_router_grad without a device");
    if (tokens == 0) return DDP_OK;
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    RouteGradArgs a{};
    a.logits = static_cast<const char*>(logits);
    a.dweights = static_cast<const char*>(dweights);
    a.experts_in = experts_in;
    a.dlogits = static_cast<char*>(dlogits);
    a.tokens = tokens;
    a.stride = stride;
    a.dstride = dlogits_stride;
    a.experts = h->experts;
    a.chosen = h->chosen;
    a.score = h->score;
    a.renormalise = h->renormalise;
    a.dweights_type = dweights_dtype;
    a.scale = h->scale;
    LAYER_HIP(h, dtype == DDP_FP32 ? launch_grad<DDP_FP32>(h, a) : dtype == DDP_FP16 ? launch_grad<DDP_FP16>(h, a) : launch_grad<DDP_BF16>(h, a));
    return DDP_OK;
}

int32_t ddp_router_balance(ddp_router* h, int32_t replicas, const int32_t* counts, float rate, const float* bias, float* bias_out) {
    if (!h) return DDP_ERR_ARG;
    if (replicas < 1 || replicas > DDP_MAX_REPLICAS) return layer_fail(h, DDP_ERR_ARG, "ddp_router_balance: replicas outside [1, DDP_MAX_REPLICAS]");
    if (!counts || !bias || !bias_out) return layer_fail(h, DDP_ERR_ARG, "ddp_router_balance: null pointer");
    if (misaligned(counts, 4) || misaligned(bias, 4) || misaligned(bias_out, 4)) return layer_fail(h, DDP_ERR_ARG, "ddp_router_balance: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_router_balance without a device");
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    hipLaunchKernelGGL(balance_kernel, dim3(1), dim3(kMaxExperts), 0, h->stream, counts, replicas, h->experts, rate, bias, bias_out);
    LAYER_HIP(h, hipGetLastError());
    return DDP_OK;
}

}  // extern "C"
