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
    float scale;
};
struct RouteGradArgs {
    const char *logits, *dweights;
    const int32_t* experts_in;
    char* dlogits;
    int64_t tokens, stride, dstride;
    int32_t experts, chosen, score, renormalise, dweights_type;
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

constexpr double kNone = -__builtin_huge_val();

// A wave a token, EACH experts a lane, in binary64.
template <int LT, int EACH>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    extern __shared__ int32_t counts[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (a.counts != nullptr) {
        for (int e = threadIdx.x; e < a.experts; e += kThreads) counts[e] = 0;
        __syncthreads();
    }
    const int per_group = a.experts / a.groups;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * kWaves) {
        double s[EACH], key[EACH];
        float x[EACH], largest = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = i * 64 + lane;
            x[i] = e < a.experts ? load_one<LT>(a.logits + (t * a.stride + e) * ElemBytes<LT>::value) : -__builtin_huge_valf();
            largest = fmaxf(largest, x[i]);
        }
        if (a.score == DDP_SCORE_SOFTMAX) {
            largest = wave_max(largest);
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s[i] = x[i] == -__builtin_huge_valf() ? 0.0 : exp(static_cast<double>(x[i]) - largest);
                sum += s[i];
            }
            sum = wave_sum(sum);
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] /= sum;
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] = 1.0 / (1.0 + exp(-static_cast<double>(x[i])));
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = i * 64 + lane;
            key[i] = e < a.experts ? s[i] + (a.bias != nullptr ? static_cast<double>(a.bias[e]) : 0.0) : kNone;
            if (x[i] == -__builtin_huge_valf() || !(key[i] > kNone)) key[i] = kNone;          // (NaN too)
        }
        if (a.kept < a.groups) {
            double rank = kNone;                     // lane g: of group g
            for (int g = 0; g < a.groups; ++g) {
                double sum = kNone;
                int used = -1;
                for (int n = 0; n < a.top; ++n) {
                    double k = kNone;
                    int at = kMaxExperts;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        const int e = i * 64 + lane;
                        if (e / per_group == g && e != used && key[i] > k) {
                            k = key[i];
                            at = e;
                        }
                    }
                    wave_best(k, at);
                    if (k > kNone) sum = n == 0 ? k : sum + k;
                    used = at;
                }
                if (lane == g) rank = sum;
            }
            uint64_t open = 0;
            for (int n = 0; n < a.kept; ++n) {
                double k = rank;
                int at = lane;
                wave_best(k, at);
                if (!(k > kNone)) break;
                open |= uint64_t(1) << at;
                if (lane == at) rank = kNone;
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int e = i * 64 + lane;
                if (e < a.experts && !(open >> (e / per_group) & 1)) key[i] = kNone;
            }
        }
        double mine = 0.0, sum = 0.0;                // lane n: of the n-th choice
        int expert = -1;
        for (int n = 0; n < a.chosen; ++n) {
            double k = kNone;
            int at = kMaxExperts;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (key[i] > k) {
                    k = key[i];
                    at = i * 64 + lane;
                }
            wave_best(k, at);
            if (!(k > kNone)) break;
            double w = 0.0;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (at == i * 64 + lane) {
                    w = s[i];
                    key[i] = kNone;
                }
            w = __shfl(w, at & 63);
            sum += w;
            if (lane == n) {
                mine = w;
                expert = at;
            }
        }
        if (lane < a.chosen) {
            double w = mine * a.scale;
            if (a.renormalise) w = sum > 0.0 ? w / sum : 0.0;
            a.experts_out[t * a.chosen + lane] = expert;
            store_weight(a.weights, a.weights_type, t * a.chosen + lane, static_cast<float>(w));
            if (a.counts != nullptr && expert >= 0) atomicAdd(&counts[expert], 1);
        }
    }
    if (a.counts == nullptr) return;
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kThreads)
        if (counts[e] != 0) atomicAdd(a.counts + e, counts[e]);
}

__global__ __launch_bounds__(kThreads) void clear_kernel(int32_t* counts, int n) {
    for (int e = threadIdx.x; e < n; e += kThreads) counts[e] = 0;
}

template <int LT, int EACH>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteGradArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * kWaves) {
        float s[EACH], d[EACH] = {}, largest = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = i * 64 + lane;
            s[i] = e < a.experts ? load_one<LT>(a.logits + (t * a.stride + e) * ElemBytes<LT>::value) : -__builtin_huge_valf();
            largest = fmaxf(largest, s[i]);
        }
        if (a.score == DDP_SCORE_SOFTMAX) {
            largest = wave_max(largest);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                s[i] = s[i] == -__builtin_huge_valf() ? 0.0f : expf(s[i] - largest);
                sum += s[i];
            }
            sum = wave_sum(sum);
#pragma unroll
            for (int i = 0; i < EACH; ++i) s[i] /= sum;
        }
        float left[EACH];                            // 1 - s of the sigmoid, without the difference
        if (a.score == DDP_SCORE_SIGMOID) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const float x = s[i], z = expf(-fabsf(x)), big = 1.0f / (1.0f + z), small = z / (1.0f + z);
                s[i] = x < 0.0f ? small : big;
                left[i] = x < 0.0f ? big : small;
                if (x != x) s[i] = left[i] = x;
            }
        }
        // lane n: the n-th choice
        const int expert = lane < a.chosen ? a.experts_in[t * a.chosen + lane] : -1;
        const bool named = expert >= 0 && expert < a.experts;
        float w = 0.0f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float v = __shfl(s[i], expert & 63);
            if (named && expert >> 6 == i) w = v;
        }
        float g = named ? load_weight(a.dweights, a.dweights_type, t * a.chosen + lane) * a.scale : 0.0f;
        if (a.renormalise) {
            const float sum = wave_sum(w), dot = wave_sum(g * w);
            g = named && sum > 0.0f ? (g - dot / sum) / sum : 0.0f;
        }
        const float dot = a.score == DDP_SCORE_SOFTMAX ? wave_sum(g * w) : 0.0f;
        const bool any = __ballot(named) != 0;
        for (int n = 0; n < a.chosen; ++n) {
            const int e = __shfl(expert, n);
            const float v = __shfl(g, n);
            if (e < 0 || e >= a.experts) continue;
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (e == i * 64 + lane) d[i] += v;
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int e = i * 64 + lane;
            float x = a.score == DDP_SCORE_SOFTMAX ? s[i] * (d[i] - dot) : d[i] * s[i] * left[i];
            if (!any) x = 0.0f;
            if (e < a.experts) store_one<LT>(a.dlogits + (t * a.dstride + e) * ElemBytes<LT>::value, x);
        }
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

template <int LT, int EACH>
hipError_t launch_route(ddp_router* h, const RouteArgs& a, unsigned blocks) {
    hipLaunchKernelGGL((route_kernel<LT, EACH>), dim3(blocks), dim3(kThreads), a.counts != nullptr ? static_cast<size_t>(a.experts) * 4 : 0, h->stream, a);
    return hipGetLastError();
}
template <int LT, int EACH>
hipError_t launch_route(ddp_router* h, const RouteGradArgs& a, unsigned blocks) {
    hipLaunchKernelGGL((route_grad_kernel<LT, EACH>), dim3(blocks), dim3(kThreads), 0, h->stream, a);
    return hipGetLastError();
}
template <int LT, typename Args>
hipError_t launch_each(ddp_router* h, const Args& a, unsigned blocks) {
    if (a.experts <= 64) return launch_route<LT, 1>(h, a, blocks);
    if (a.experts <= 128) return launch_route<LT, 2>(h, a, blocks);
    if (a.experts <= 256) return launch_route<LT, 4>(h, a, blocks);
    if (a.experts <= 512) return launch_route<LT, 8>(h, a, blocks);
    return launch_route<LT, 16>(h, a, blocks);
}
template <typename Args>
hipError_t launch_typed(ddp_router* h, const Args& a, int dtype) {
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, kBlocks));
    if (dtype == DDP_FP32) return launch_each<DDP_FP32>(h, a, blocks);
    if (dtype == DDP_FP16) return launch_each<DDP_FP16>(h, a, blocks);
    return launch_each<DDP_BF16>(h, a, blocks);
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
    LAYER_HIP(h, launch_typed(h, a, dtype));
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
    LAYER_HIP(h, launch_typed(h, a, dtype));
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
