// Routing of tokens to experts, its gradient, and the step of the balance bias.
//
//   s = softmax(logits) or sigmoid(logits),  key = s + bias
//   a group's score is the sum of its `top` largest keys; the experts of the `kept` best groups are open
//   the `chosen` largest open keys, descending, ties to the lower index;  w = scale s (/ the sum of the chosen s)
//   gradient: t = dw scale, renormalised (t - sum t w') / sum s;  softmax: s (t - sum t s),  sigmoid: t s (1 - s)
//
// 65536 tokens of 256 binary32 logits, eight of four groups of eight (71 MB): 47 us with the balance step, where the bytes alone would take 11.
// Choices have to be those of binary64, so this is bound by vector instructions (30 us: 966 of a wave for four tokens) and then by the
// latency of the tokens that binary32 leaves open (12) and of the balance step's launch (4.5).  The gradient, 15 us, waits for chains of three loads.
#include "layer_host.h"

struct ddp_router : ddp::LayerHandle {
    int32_t* copies = nullptr;                   // [kCopies][experts] counts, zeros between calls
    int32_t experts = 0, chosen = 0, groups = 0, kept = 0, top = 0, score = 0, renormalise = 0;
    float scale = 1.0f;
};

namespace {

using namespace ddp;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxExperts = 1024, kMaxChosen = 64, kMaxGroups = 64;
constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int kCopies = 16;

struct RouteArgs {
    const char* logits;
    const float* bias;
    int32_t* experts_out;
    char* weights;
    int32_t *counts, *copies;
    int64_t tokens, stride;
    int32_t experts, chosen, groups, kept, top, score, renormalise, weights_type, accumulate;
    int32_t log2_lanes, each, log2_group, listed;    // of a team: lanes, experts a lane, lanes a group, candidates
    int32_t room;                                    // keys (or a lane's sorted words) in LDS for each wave
    float scale;
};
struct RouteGradArgs {
    const char *logits, *dweights;
    const int32_t* experts_in;
    char* dlogits;
    int64_t tokens, stride, dstride;
    int32_t experts, chosen, score, renormalise, dweights_type, log2_lanes, stream;
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
template <int CTRL>
__device__ __forceinline__ double lane_moved(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b), CTRL, 0xF, 0xF, true));
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(b >> 32), CTRL, 0xF, 0xF, true));
    return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_max(double x) {
    x = fmax(x, lane_moved<0xB1>(x));                // quad_perm: 1 0 3 2
    x = fmax(x, lane_moved<0x4E>(x));                // quad_perm: 2 3 0 1
    x = fmax(x, lane_moved<0x141>(x));               // row_half_mirror
    x = fmax(x, lane_moved<0x140>(x));               // row_mirror
    x = fmax(x, __shfl_xor(x, 16));
    return fmax(x, __shfl_xor(x, 32));
}
// The largest key and the lowest index that has it.
__device__ __forceinline__ void wave_best(double& key, int& at) {
    const double top = wave_max(key);
    uint64_t here = __ballot(key == top);
    key = top;
    int lowest = __builtin_amdgcn_readlane(at, __ffsll(static_cast<unsigned long long>(here)) - 1);
    for (here &= here - 1; here != 0; here &= here - 1) lowest = min(lowest, __builtin_amdgcn_readlane(at, __ffsll(static_cast<unsigned long long>(here)) - 1));
    at = lowest;
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
//
// The plain way, some 10 us a token and 434 us for 65536 of 256 experts.

// keys: of the experts, in LDS.
template <int LT>
__device__ __forceinline__ void route_token(const RouteArgs& a, int64_t t, double* keys, int32_t* counts) {
    const int lane = threadIdx.x & 63, per_group = a.experts / a.groups;
    const char* row = a.logits + t * a.stride * ElemBytes<LT>::value;
    auto logit = [&](int e) { return load_one<LT>(row + e * ElemBytes<LT>::value); };
    const bool softmax = a.score == DDP_SCORE_SOFTMAX;
    float largest = 0.0f;
    double sum = 1.0;
    if (softmax) {
        largest = kMasked;
        for (int e = lane; e < a.experts; e += 64) largest = fmaxf(largest, logit(e));
        largest = wave_max(largest);
        sum = 0.0;
    }
    // exp(x - largest) of a softmax, 1 + exp(-x) of a sigmoid
    auto part = [&](float x) { return softmax ? (x == kMasked ? 0.0 : exp(static_cast<double>(x) - largest)) : 1.0 + exp(-static_cast<double>(x)); };
    auto score = [&](double part) { return softmax ? part / sum : 1.0 / part; };
#pragma unroll 1
    for (int e = lane; e < a.experts; e += 64) {
        keys[e] = part(logit(e));
        if (softmax) sum += keys[e];
    }
    if (softmax) sum = wave_sum(sum);
    for (int e = lane; e < a.experts; e += 64) {
        const double key = score(keys[e]) + (a.bias != nullptr ? static_cast<double>(a.bias[e]) : 0.0);
        keys[e] = logit(e) != kMasked && key > kNone ? key : kNone;       // (NaN is not above)
    }
    wave_meets();
    uint64_t open = ~uint64_t(0);
    if (a.kept < a.groups) {
        double first = kNone, second = kNone;        // lane g: of group g
        if (lane < a.groups) {
#pragma unroll 4
            for (int i = 0; i < per_group; ++i) {
                const double k = keys[lane * per_group + i];
                second = fmax(fmin(first, k), second);
                first = fmax(first, k);
            }
            if (a.top == 2 && second > kNone) first += second;
        }
        open = 0;
        for (int n = 0; n < a.kept; ++n) {
            double k = first;
            int at = lane;
            wave_best(k, at);
            if (!(k > kNone)) break;
            open |= uint64_t(1) << at;
            if (lane == at) first = kNone;
        }
        for (int e = lane; e < a.experts; e += 64)
            if (!(open >> (e / per_group) & 1)) keys[e] = kNone;
    }
    double best = kNone;                             // of the lane's keys
    int best_at = kMaxExperts;
    auto find = [&]() {
        best = kNone;
        best_at = kMaxExperts;
#pragma unroll 4
        for (int e = lane; e < a.experts; e += 64)
            if (keys[e] > best) {
                best = keys[e];
                best_at = e;
            }
    };
    find();
    int expert = -1;                                 // lane n: the n-th choice
    for (int n = 0; n < a.chosen; ++n) {
        double k = best;
        int at = best_at;
        wave_best(k, at);
        if (!(k > kNone)) break;
        if (lane == n) expert = at;
        if (at == best_at) {
            keys[at] = kNone;
            find();
        }
    }
    double w = lane < a.chosen && expert >= 0 ? score(part(logit(expert))) : 0.0;
    const double all = wave_sum(w);
    if (lane < a.chosen) {
        w *= a.scale;
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
// A block alone writes the counts.  More blocks add theirs to copies, which the next kernel sums: 2048 blocks of 256 experts at
// one copy took 30 us longer.
template <bool ALONE>
__device__ __forceinline__ void add_counts(const RouteArgs& a, const int32_t* counts) {
    if (a.counts == nullptr) return;
    __syncthreads();
    if (ALONE && gridDim.x == 1) {
        for (int e = threadIdx.x; e < a.experts; e += kThreads) a.counts[e] = counts[e] + (a.accumulate ? a.counts[e] : 0);
        return;
    }
    int32_t* to = a.copies + blockIdx.x % kCopies * a.experts;
    for (int e = threadIdx.x; e < a.experts; e += kThreads)
        if (counts[e] != 0) atomicAdd(to + e, counts[e]);
}
// The sum of an expert's copies, and zeros in them for the next call.
__device__ __forceinline__ int32_t take_copies(int32_t* copies, int experts, int e) {
    int32_t x[kCopies], sum = 0;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) x[c] = copies[c * experts + e];
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
        sum += x[c];
        if (x[c] != 0) copies[c * experts + e] = 0;
    }
    return sum;
}

// All tokens (where no team's lanes divide into the groups), or those that teams have left.
constexpr int32_t kAgain = -2;
template <int LT, bool ALL>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    extern __shared__ double keys[];                 // [kWaves][experts], then the counts
    int32_t* counts = reinterpret_cast<int32_t*>(keys + kWaves * a.experts);
    clear_counts(a, counts);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    double* mine = keys + wave * a.experts;
    if constexpr (ALL) {
        for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * kWaves) route_token<LT>(a, t, mine, counts);
    } else {
        for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * 64; t0 < a.tokens; t0 += static_cast<int64_t>(gridDim.x) * 64) {
            const bool left = t0 + lane < a.tokens && a.experts_out[(t0 + lane) * a.chosen] == kAgain;
            __syncthreads();                         // (all waves look before one of them is done with a token)
            int n = 0;
            for (uint64_t some = __ballot(left); some != 0; some &= some - 1, ++n)
                if (n % kWaves == wave) route_token<LT>(a, t0 + __ffsll(static_cast<unsigned long long>(some)) - 1, mine, counts);
        }
    }
    if constexpr (ALL) {
        add_counts<true>(a, counts);
    } else if (a.counts != nullptr) {                // the teams' kernel has cleared the counts, where they are not added to
        __syncthreads();
        for (int e = threadIdx.x; e < a.experts; e += kThreads) {
            const int32_t n = counts[e] + (e % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x) ? take_copies(a.copies, a.experts, e) : 0);
            if (n != 0) atomicAdd(a.counts + e, n);
        }
    }
}

// ---- a token by a team ----
//
// A team of 1 to 64 lanes has up to kEach neighbouring experts a lane.  Keys in binary32 become words that sort as they do, with the place
// in the lane for their last four bits; a lane sorts its own, and the team takes the largest head, as often as there are candidates: one more than
// are chosen.  Where the candidates' keys are all further apart than the error of a binary32 key, their order is that of binary64.
// Where not, the candidates are ordered again by whole binary32 keys, equal logits with equal biases by their index.  Where that too leaves it open, or the
// groups' scores come near each other, a wave does the token over in binary64: of 256 normal logits of deviation 1.5 in eight groups, one token in 400.
// The errors are taken from the largest score and bias of all experts, so that small keys count as near each other too: with logits of deviation 5
// most tokens are done over (65536 x 256, softmax with small biases: 43 us at 1.5, 76 at 3, 203 at 5, 255 at 8), with a finite mask in the bias
// all of them (252), and so are those whose logits are all equal, which take the longest (653).

constexpr int kEach = 16, kSpare = 1;                // (two spare candidates: 65536 x 256 48.7 us against 47.7, 86976 x 143 66.7 against 64.3)
// A key's error in parts of 2^-24 of the largest score and bias: exp, sum and quotient of a softmax over 1024 under 30, the key's
// rounding and the lift's 6 (a lifted key is up to twice as large), the bits given to the place 64: two keys 200.
constexpr float kApart = 0x1p-16f;
// The same of whole keys: 30 of the largest score and 3 of score and bias each of a softmax, 5 of a sigmoid.
constexpr float kNearSoftmax = 0x1p-18f, kNearKey = 0x1p-20f;
// Chosen scores whose sum is below this (biases have chosen them, or every logit of a sigmoid is far below 0) are near binary32's end, their
// quotients not: a wave takes the weights in binary64.  (Next to a larger sum a chosen score below 2^-126 loses its bits: less than 2^-26 of that.)
constexpr float kTiny = 0x1p-100f;
// Below this a lifted key and the sum of a group's two largest are finite, above -inf and below inf.
constexpr float kGroupLift = 0x1p126f;

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
    if (log2 > 4) f([](uint32_t x) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    });
    if (log2 > 5) f([](uint32_t x) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    });
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

// The first lane of a team that is in the mask (one is).
__device__ __forceinline__ int first_lane(uint64_t mask, int log2_lanes, int of_team0) {
    if (log2_lanes == 6) return __ffsll(static_cast<unsigned long long>(mask)) - 1;
    const uint32_t half = of_team0 & 32 ? static_cast<uint32_t>(mask >> 32) : static_cast<uint32_t>(mask);
    return __ffs(static_cast<int>(half >> (of_team0 & 31))) - 1;
}

// A key as a word: positive floats sort as their bits do, so `lift` makes the key positive; 0: no key.
__device__ __forceinline__ float key_of(uint32_t word, float lift) { return as_float(word & ~15u) - lift; }

// Descending, by Batcher's odd-even merges.
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

// EACH: the lane's experts, a.each of them used.  LANES: the logarithm of a team's lanes, if it is known (the steps of a meeting need no branches then:
// 65536 tokens of 256 experts 47 us without).  Four lanes and 64 are held to the 80 registers of six waves, which the compiler exceeds by one.
template <int LT, int EACH, bool HERE, int LANES>
__global__ __launch_bounds__(kThreads, !HERE && (LANES == 2 || LANES == 6) ? 6 : 1) void route_team_kernel(RouteArgs a) {
    extern __shared__ double keys[];                 // [kWaves][room], then candidates and counts
    const int log2_lanes = LANES >= 0 ? LANES : a.log2_lanes, lanes = 1 << log2_lanes, l = threadIdx.x & (lanes - 1), team = threadIdx.x >> log2_lanes, teams = kThreads >> log2_lanes;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    char* behind = reinterpret_cast<char*>(keys + kWaves * a.room);
    uint32_t* word = reinterpret_cast<uint32_t*>(behind) + team * a.listed;          // of each candidate: its key, then its weight
    int32_t* at = reinterpret_cast<int32_t*>(behind) + (teams + team) * a.listed;    // its expert, or -1
    int32_t* place = reinterpret_cast<int32_t*>(behind) + (2 * teams + team) * a.listed;      // its rank, once ordered
    float* lifted = reinterpret_cast<float*>(behind) + 3 * teams * a.listed;
    int32_t* counts = reinterpret_cast<int32_t*>(behind) + 3 * teams * a.listed + max(EACH << log2_lanes, kWaves);
    uint32_t* sorted = reinterpret_cast<uint32_t*>(keys + wave * a.room) + lane;     // the lane's words, 64 apart
    clear_counts(a, counts);
    const int e0 = l * a.each, mine = max(min(a.experts - e0, a.each), 0);
    if (!HERE && a.counts != nullptr && !a.accumulate && blockIdx.x == 0)
        for (int e = threadIdx.x; e < a.experts; e += kThreads) a.counts[e] = 0;
    // biases, lifted, in LDS: the i-th of a team's lanes side by side (in registers they would cost a wave in six)
    float of_bias = 0.0f;
    for (int e = threadIdx.x; a.bias != nullptr && e < a.experts; e += kThreads) {
        const float x = fabsf(a.bias[e]);
        of_bias = fmaxf(of_bias, x < __builtin_huge_valf() ? x : 0.0f);
    }
    of_bias = team_max(6, of_bias);
    if (lane == 0) lifted[wave] = of_bias;
    __syncthreads();
    of_bias = fmaxf(fmaxf(lifted[0], lifted[1]), fmaxf(lifted[2], lifted[3]));
    static_assert(kWaves == 4, "");
    const float lift = of_bias * (1.0f + 0x1p-20f) + 0x1p-60f;       // (above every -bias)
    __syncthreads();
    for (int i = threadIdx.x; i < EACH << log2_lanes; i += kThreads) {
        const int of = i & (lanes - 1), k = i >> log2_lanes, e = of * a.each + k;
        lifted[i] = k < a.each && e < a.experts ? (a.bias != nullptr ? a.bias[e] : 0.0f) + lift : kMasked;
    }
    __syncthreads();
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
            largest = team_max(log2_lanes, largest);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s[i] = x[i] == kMasked ? 0.0f : fast_exp(x[i] - largest);
                sum += s[i];
            }
            sum = team_sum(log2_lanes, sum);
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
            const float key = s[i] + lifted[(i << log2_lanes) + l];
            w[i] = x[i] != kMasked && key > 0.0f ? (as_bits(key) & ~15u) | static_cast<uint32_t>(15 - i) : 0u;
        }
        sort_words<EACH>(w);
        bool again = false;                          // the token is for a wave
        const int of_team0 = lane & ~(lanes - 1);
        if (a.kept < a.groups) {
            float first = w[0] != 0 ? key_of(w[0], lift) : kMasked, second = kMasked;
            if constexpr (EACH > 1) second = w[1] != 0 ? key_of(w[1], lift) : kMasked;
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
            const float worst = -team_max(log2_lanes, before < a.kept && group < a.groups ? -rank : kMasked);
            const float next = team_max(log2_lanes, before >= a.kept && group < a.groups ? rank : kMasked);
            // (a finite bias of 2^126 and more takes a lifted key, or a group's two keys together, out of binary32: binary64)
            again = (next > kMasked && !(worst - next > 2.0f * apart)) || !(lift < kGroupLift);
            if (before >= a.kept) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) w[i] = 0;
            }
        }
        // what is behind a lane's head: in LDS, or where latency counts and there is little, in registers
        constexpr bool SHIFT = HERE && EACH <= 8;
        if constexpr (!SHIFT) {
#pragma unroll
            for (int i = 1; i < EACH; ++i) sorted[i * 64] = w[i];
        }
        float left = kMasked;                        // the largest key behind the candidates
        int taken = 0;
        for (int n = 0; n <= a.listed; ++n) {
            const uint32_t head = w[0] >> 4, top = team_max(log2_lanes, head);
            if (n == a.listed) {
                if (top != 0) left = key_of(top << 4, lift);
                break;
            }
            if (first_lane(__ballot(head == top), log2_lanes, of_team0) == l) {
                word[n] = w[0];
                at[n] = top != 0 ? e0 + 15 - static_cast<int>(w[0] & 15u) : -1;
                if constexpr (SHIFT) {
#pragma unroll
                    for (int i = 1; i < EACH; ++i) w[i - 1] = w[i];
                    w[EACH - 1] = 0u;
                } else {
                    ++taken;
                    w[0] = taken < EACH ? sorted[taken * 64] : 0u;
                }
            }
        }
        wave_meets();
        // candidates go round the lanes: are two of the first a.chosen + 1 too near each other?
        bool near = false;
        for (int n = l; n < a.chosen; n += lanes) {
            const uint32_t here = word[n], behind = n + 1 < a.listed ? word[n + 1] : 0u;
            if (here != 0 && (behind != 0 || n + 1 >= a.listed)) {
                const float k = key_of(here, lift), b = n + 1 < a.listed ? key_of(behind, lift) : left;
                near |= b != kMasked && !(k - b > apart);       // (a lift beyond binary32 makes NaN of them)
            }
        }
        const uint64_t of_team = lanes == 64 ? ~uint64_t(0) : (uint64_t(1) << lanes) - 1;
        const bool close = (__ballot(near) >> of_team0 & of_team) != 0;
        const bool ordered = __ballot(close && live && !again) != 0;
        auto logit = [&](int e) { return load_one<LT>(row + e * ElemBytes<LT>::value); };
        auto score = [&](float x) { return a.score == DDP_SCORE_SOFTMAX ? expf(x - largest) * most : 1.0f / (1.0f + expf(-x)); };
        auto bias_of = [&](int e) { return a.bias != nullptr ? a.bias[e] : 0.0f; };
        if (ordered) {                               // the candidates once more, by whole keys
            for (int n = l; n < a.listed; n += lanes)
                if (at[n] >= 0) word[n] = as_bits(score(logit(at[n])) + bias_of(at[n]));
            wave_meets();
            const float same = (a.score == DDP_SCORE_SOFTMAX ? kNearSoftmax * most : 0.0f) + kNearKey * (most + of_bias);
            for (int n = l; n < a.listed; n += lanes) {
                const int e = at[n];
                if (e < 0) continue;
                const float key = as_float(word[n]);
                int rank = 0;
                for (int m = 0; m < a.listed; ++m) {
                    const int o = at[m] & 0xFFFF;
                    if (at[m] < 0 || m == n) continue;
                    const float other = as_float(word[m]);
                    rank += other > key || (other == key && o < e);
                    // equal for certain where logit and bias are
                    if (!(fabsf(other - key) > same)) again |= logit(o) != logit(e) || bias_of(o) != bias_of(e);
                }
                if (rank < a.chosen) again |= left != kMasked && !(key - left > apart);
                place[n] = rank;
            }
            again = (__ballot(again) >> of_team0 & of_team) != 0;
        }
        if (live && !again) {
            float all = 0.0f;
            for (int n = l; n < a.listed; n += lanes) {
                const int e = at[n], rank = ordered && e >= 0 ? place[n] : n;
                float v = 0.0f;
                if (rank < a.chosen && e >= 0) v = score(logit(e));
                all += v;
                word[n] = as_bits(v);
                at[n] = rank < a.chosen ? (e < 0 ? -1 : e | rank << 16) : -2;
                if (rank < a.chosen && e < 0) {
                    a.experts_out[t * a.chosen + rank] = -1;
                    store_weight(a.weights, a.weights_type, t * a.chosen + rank, 0.0f);
                }
            }
            all = team_sum(log2_lanes, all);
            if (all < kTiny) {
                wave_meets();
                again = at[0] != -1;                 // some are chosen
            }
            const float factor = !a.renormalise ? 1.0f : all > 0.0f ? 1.0f / all : 0.0f;      // (scale / all may leave binary32)
            for (int n = l; n < a.listed; n += lanes) {
                if (again || at[n] < 0) continue;
                const int e = at[n] & 0xFFFF, rank = at[n] >> 16;
                a.experts_out[t * a.chosen + rank] = e;
                store_weight(a.weights, a.weights_type, t * a.chosen + rank, as_float(word[n]) * factor * a.scale);
                if (a.counts != nullptr) atomicAdd(&counts[e], 1);
            }
        }
        if constexpr (HERE) {
            for (uint64_t left_over = __ballot(live && again && l == 0); left_over != 0; left_over &= left_over - 1) {
                const int which = __ffsll(static_cast<unsigned long long>(left_over)) - 1;
                wave_meets();
                route_token<LT>(a, base + ((static_cast<int>(threadIdx.x & ~63u) + which) >> log2_lanes), keys + wave * a.room, counts);
            }
        } else {
            if (live && again && l == 0) a.experts_out[t * a.chosen] = kAgain;
        }
        wave_meets();
    }
    add_counts<HERE>(a, counts);
}

__global__ __launch_bounds__(64) void count_kernel(int32_t* copies, int32_t* counts, int experts, int accumulate) {
    const int e = blockIdx.x * 64 + threadIdx.x;
    if (e < experts) counts[e] = take_copies(copies, experts, e) + (accumulate ? counts[e] : 0);
}

// The largest number of binary32 whose sigmoid is 0 in binary64 too (exp(-x) is beyond it), as its weight is.
constexpr float kNoScore = -709.78271484375f;

// A token's gradient by a team of lanes with EACH experts each, in vectors of 16 bytes side by side.  What the chosen experts get is put together in a row in LDS, which is zeros
// otherwise, and everyone reads what is theirs.  Only a softmax that is not renormalised reads the other logits: renormalised, it is that of the
// chosen ones, and 64 bits or 32 leave nothing to the rest.  Renormalised scores are taken with a common factor exp(-shift) that makes the largest
// 1 (a sigmoid's at least 1/2), so that small ones do not leave the range of binary32 before they are divided.
template <int LT, int EACH, bool WHOLE>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteGradArgs a) {
    extern __shared__ float lds[];                   // [teams]: the row, then of the chosen: gradient, score, expert
    const int lanes = 1 << a.log2_lanes, l = threadIdx.x & (lanes - 1), team = threadIdx.x >> a.log2_lanes, teams = kThreads >> a.log2_lanes;
    constexpr int N = EACH * ElemBytes<LT>::value >= 16 ? 16 / ElemBytes<LT>::value : EACH, V = EACH / N;
    float* row = lds + team * (lanes * EACH + 3 * a.chosen);
    float* of = row + lanes * EACH;
    float* score = of + a.chosen;
    int32_t* at = reinterpret_cast<int32_t*>(score + a.chosen);
#pragma unroll
    for (int i = 0; i < EACH; ++i) row[l * EACH + i] = 0.0f;
    auto first = [&](int v) { return (v * lanes + l) * N; };             // of a vector's experts
    auto have = [&](int v) { return max(min(a.experts - first(v), N), 0); };
    const int of_team0 = static_cast<int>(threadIdx.x & 63) & ~(lanes - 1);
    const uint64_t of_team = lanes == 64 ? ~uint64_t(0) : (uint64_t(1) << lanes) - 1;
    const bool sigmoid = !WHOLE && a.score == DDP_SCORE_SIGMOID, renormalise = !WHOLE && a.renormalise;
    // a lane's first choice of the next token is on the way while this one's logit is
    int next_expert = -1;
    float next_weight = 0.0f;
    auto fetch = [&](int64_t t) {
        const bool some = t < a.tokens && l < a.chosen;
        const int64_t from = some ? t * a.chosen + l : 0;
        next_expert = a.experts_in[from];
        next_weight = load_weight(a.dweights, a.dweights_type, from);
        if (!some) next_expert = -1;
    };
    fetch(static_cast<int64_t>(blockIdx.x) * teams + team);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * teams; base < a.tokens; base += static_cast<int64_t>(gridDim.x) * teams) {
        const int64_t t = base + team;
        const bool live = t < a.tokens;
        const int expert = next_expert;
        const float weight = next_weight;
        float logit = 0.0f;
        fetch(t + static_cast<int64_t>(gridDim.x) * teams);
        const char* from = a.logits + t * a.stride * ElemBytes<LT>::value;
        float s[V][N], largest = 0.0f, part = 0.0f;
        if constexpr (WHOLE) {
#pragma unroll
            for (int v = 0; v < V; ++v) load_some<LT, N>(from + first(v) * ElemBytes<LT>::value, live ? have(v) : 0, s[v]);
            largest = kMasked;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (i >= have(v)) s[v][i] = kMasked;
                    largest = fmaxf(largest, s[v][i]);
                }
            largest = team_max(a.log2_lanes, largest);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    s[v][i] = s[v][i] == kMasked ? 0.0f : expf(s[v][i] - largest);
                    part += s[v][i];
                }
            part = 1.0f / team_sum(a.log2_lanes, part);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) s[v][i] *= part;
        }
        // the chosen go round the lanes
        bool any = false;
        float most = kMasked, all = 0.0f, dot = 0.0f;
        for (int n = l; n < a.chosen; n += lanes) {
            const int e = n == l ? expert : live ? a.experts_in[t * a.chosen + n] : -1;
            const bool named = e >= 0 && e < a.experts;
            float x = kMasked, g = 0.0f;
            if (named) {
                x = load_one<LT>(from + e * ElemBytes<LT>::value);
                if (n == l) logit = x;
                g = (n == l ? weight : load_weight(a.dweights, a.dweights_type, t * a.chosen + n)) * a.scale;
            }
            any |= named;
            most = fmaxf(most, x);
            at[n] = named ? e : -1;
            of[n] = g;
            score[n] = x;
        }
        const float factor = WHOLE ? part : 1.0f, none = sigmoid ? kNoScore : kMasked;
        float shift = WHOLE ? largest : 0.0f;
        if (renormalise) {
            most = team_max(a.log2_lanes, most);
            shift = sigmoid ? fminf(most, 0.0f) : most;
        }
        for (int n = l; n < a.chosen; n += lanes) {
            const float x = score[n];
            float w = 0.0f;
            if (!(x <= none)) w = sigmoid && x > 0.0f ? 1.0f / (1.0f + expf(-x)) : expf(x - shift) * (sigmoid ? factor / (1.0f + expf(x)) : factor);
            all += w;
            dot += of[n] * w;
            score[n] = w;
        }
        if (renormalise) {
            all = team_sum(a.log2_lanes, all);
            dot = team_sum(a.log2_lanes, dot);
            const float mean = dot / all;
            for (int n = l; n < a.chosen; n += lanes) of[n] = score[n] != 0.0f ? (of[n] - mean) * (score[n] / all) : 0.0f;
        } else if (sigmoid) {
            for (int n = l; n < a.chosen; n += lanes) of[n] *= score[n];
        } else {
            any = (__ballot(any) >> of_team0 & of_team) != 0;
            dot = team_sum(a.log2_lanes, dot);
        }
        wave_meets();
        for (int n = l; n < a.chosen; n += lanes) {
            const int e = at[n];
            if (e < 0) continue;
            float sum = 0.0f;                        // (an expert that is named twice)
            for (int m = 0; m < a.chosen; ++m) {
                const float one = of[m];             // (no condition on the read: it would be waited for)
                sum += at[m] == e ? one : 0.0f;
            }
            if (sigmoid) {
                const float x = n == l ? logit : load_one<LT>(from + e * ElemBytes<LT>::value);
                sum *= 1.0f / (1.0f + expf(x));                  // 1 - s, without the difference
            }
            row[e] = sum;
        }
        wave_meets();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                d[i] = row[first(v) + i];
                if (WHOLE) d[i] = any ? s[v][i] * (d[i] - dot) : 0.0f;
            }
            char* to = a.dlogits + (t * a.dstride + first(v)) * ElemBytes<LT>::value;
            if (!live || have(v) == 0) continue;
            if (a.stream) store_some<LT, N, true>(to, have(v), d);
            else store_some<LT, N>(to, have(v), d);
        }
        wave_meets();
        for (int n = l; n < a.chosen; n += lanes)
            if (at[n] >= 0) row[at[n]] = 0.0f;
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

// Gradients of this size and more are stored past the caches (65536 x 256 16.3 us against 17.8).
constexpr int64_t kStreamBytes = int64_t(4) << 20;
// kBlocks: six waves a SIMD, all resident.  Up to kFewBlocks blocks do tokens over where they meet them: a second launch would cost more (one
// token 6.1 us against 8.6, 1270 tokens 10.9 against 11.7), but more of them would run at four waves a SIMD (65536 x 256 47.5 us against 77).
// The gradient takes kBlocks over (65536 x 256 16 us, with more blocks than that 18); other limits have not been measured.
// kFewLanes: of all teams, where tokens are few (65536: 4096 tokens 24.4 us; 262144: 27.3; 16384: 3948 tokens of 30 experts 16.6 against 14.1).
constexpr int64_t kBlocks = 1536, kFewLanes = 65536, kFewBlocks = 512;

// The team of a token: a.each experts a lane, up to `most`, so that groups have a power of two of lanes.  False: none.
bool team_of(RouteArgs& a, int most) {
    const int per_group = a.experts / a.groups;
    a.log2_lanes = a.log2_group = 0;
    if (a.kept >= a.groups) {
        a.each = std::max(std::min(most, 256 / a.chosen + 4), (a.experts + 63) / 64);        // (many candidates take more lanes: their LDS is a team's)
    } else {
        for (a.each = std::min(most, per_group); a.each > 0; --a.each) {
            const int lanes = per_group / a.each;
            if (per_group % a.each == 0 && (lanes & (lanes - 1)) == 0) break;
        }
        if (a.each == 0) return false;
        while (a.each << a.log2_group < per_group) ++a.log2_group;
    }
    while (a.each << a.log2_lanes < a.experts) ++a.log2_lanes;
    if (a.each > 8) a.log2_lanes = std::max(a.log2_lanes, 2);
    if (a.log2_lanes > 6) return false;
    a.listed = std::min(a.chosen + kSpare, a.experts);
    a.room = std::max({a.experts, 32 * (a.each > 8 ? 16 : a.each > 4 ? 8 : a.each > 2 ? 4 : a.each)});
    return true;
}
// Four lanes at least, and where tokens are few as many as find work.
bool find_team(RouteArgs& a) {
    const int64_t lanes = std::max<int64_t>(4, std::min<int64_t>(64, kFewLanes / a.tokens));
    return team_of(a, static_cast<int>(std::min<int64_t>(kEach, (a.experts + lanes - 1) / lanes))) || team_of(a, kEach);
}
// Returns whether counts are left in the copies.
template <int LT, int EACH>
bool launch_team(ddp_router* h, const RouteArgs& a, int64_t blocks, size_t bytes) {
    if (blocks <= kFewBlocks) {
        if (a.log2_lanes == 6) hipLaunchKernelGGL((route_team_kernel<LT, EACH, true, 6>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), bytes, h->stream, a);
        else hipLaunchKernelGGL((route_team_kernel<LT, EACH, true, -1>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), bytes, h->stream, a);
        return blocks > 1;
    }
    const dim3 grid(static_cast<unsigned>(std::min(blocks, kBlocks))), threads(kThreads);
    auto launch = [&](auto lanes) { hipLaunchKernelGGL((route_team_kernel<LT, EACH, false, lanes.value>), grid, threads, bytes, h->stream, a); };
    if constexpr (EACH == 16) {
        if (a.log2_lanes <= 2) launch(std::integral_constant<int, 2>());
        else if (a.log2_lanes == 3) launch(std::integral_constant<int, 3>());
        else if (a.log2_lanes == 4) launch(std::integral_constant<int, 4>());
        else if (a.log2_lanes == 5) launch(std::integral_constant<int, 5>());
        else launch(std::integral_constant<int, 6>());
    } else {
        launch(std::integral_constant<int, -1>());
    }
    const int64_t looks = (a.tokens + 63) / 64;      // tokens that a block looks through at a time
    hipLaunchKernelGGL((route_kernel<LT, false>), dim3(static_cast<unsigned>(std::min(looks, kBlocks))), dim3(kThreads),
                       static_cast<size_t>(kWaves * 8 + 4) * a.experts, h->stream, a);
    return false;
}
template <int LT>
bool launch_route(ddp_router* h, RouteArgs a) {
    if (!find_team(a)) {
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, kBlocks));
        hipLaunchKernelGGL((route_kernel<LT, true>), dim3(blocks), dim3(kThreads), static_cast<size_t>(kWaves * 8 + 4) * a.experts, h->stream, a);
        return blocks > 1;
    }
    const int teams = kThreads >> a.log2_lanes;
    const int64_t blocks = (a.tokens + teams - 1) / teams;
    const int each = a.each > 8 ? 16 : a.each > 4 ? 8 : a.each > 2 ? 4 : a.each;
    if (blocks > kFewBlocks) a.room = 32 * each;     // (no token is done over there)
    const size_t bytes = static_cast<size_t>(kWaves) * a.room * 8 + static_cast<size_t>(teams) * a.listed * 12 + static_cast<size_t>(a.experts) * 4 +
                         (std::max(each << a.log2_lanes, kWaves)) * size_t(4);
    if (a.each > 8) return launch_team<LT, 16>(h, a, blocks, bytes);
    if (a.each > 4) return launch_team<LT, 8>(h, a, blocks, bytes);
    if (a.each > 2) return launch_team<LT, 4>(h, a, blocks, bytes);
    if (a.each > 1) return launch_team<LT, 2>(h, a, blocks, bytes);
    return launch_team<LT, 1>(h, a, blocks, bytes);
}
template <int LT>
hipError_t launch_grad(ddp_router* h, RouteGradArgs a) {
    // 16 where tokens are enough for it (60 experts: 20011 tokens 7.7 us with 16 and 6.2 with 4, of 64 65536 5.4 and 9.6); many chosen take more lanes: their LDS is a team's
    int few = 0;
    while (16 << few < a.experts) ++few;
    const bool enough = a.tokens << few >= kFewBlocks * kThreads;
    const int each = a.experts > 256 || (enough && a.experts > 32 && 4 * a.chosen <= a.experts) ? 16 : 4;
    while (each << a.log2_lanes < a.experts) ++a.log2_lanes;
    const int teams = kThreads >> a.log2_lanes;
    const dim3 blocks(static_cast<unsigned>(std::min<int64_t>((a.tokens + teams - 1) / teams, kBlocks))), threads(kThreads);
    const size_t bytes = static_cast<size_t>(teams) * ((each << a.log2_lanes) + 3 * a.chosen) * 4;
    auto launch = [&](auto each, auto whole) { hipLaunchKernelGGL((route_grad_kernel<LT, each.value, whole.value>), blocks, threads, bytes, h->stream, a); };
    auto sized = [&](auto whole) {
        if (each == 16) launch(std::integral_constant<int, 16>(), whole);
        else launch(std::integral_constant<int, 4>(), whole);
    };
    if (a.score == DDP_SCORE_SOFTMAX && !a.renormalise) sized(std::true_type());
    else sized(std::false_type());
    return hipGetLastError();
}

int32_t sum_copies(ddp_router* h, int32_t* counts, int32_t accumulate) {
    hipLaunchKernelGGL(count_kernel, dim3(static_cast<unsigned>((h->experts + 63) / 64)), dim3(64), 0, h->stream, h->copies, counts, h->experts, accumulate);
    LAYER_HIP(h, hipGetLastError());
    return DDP_OK;
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
    if (device != DDP_DEVICE_NONE) {
        const int64_t bytes = static_cast<int64_t>(kCopies) * experts * 4;
        hipError_t err = layer_alloc(h, bytes);
        if (err == hipSuccess) {
            OnDevice on(device);
            err = taken(hipMemset(h->mem, 0, static_cast<size_t>(bytes)));
            if (err == hipSuccess) err = taken(hipStreamSynchronize(nullptr));
            if (err != hipSuccess) (void)taken(hipFree(h->mem));
        }
        if (err != hipSuccess) {
            delete h;
            return layer_fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        h->copies = reinterpret_cast<int32_t*>(h->mem);
    }
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
    if (tokens == 0) {
        if (!counts || accumulate) return DDP_OK;
        return sum_copies(h, counts, 0);
    }
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
    a.copies = h->copies;
    a.accumulate = accumulate != 0;
    const bool copies = dtype == DDP_FP32 ? launch_route<DDP_FP32>(h, a) : dtype == DDP_FP16 ? launch_route<DDP_FP16>(h, a) : launch_route<DDP_BF16>(h, a);
    LAYER_HIP(h, hipGetLastError());
    return counts && copies ? sum_copies(h, counts, accumulate) : DDP_OK;
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
    a.stream = tokens * h->experts * elem_bytes(dtype) >= kStreamBytes;
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
