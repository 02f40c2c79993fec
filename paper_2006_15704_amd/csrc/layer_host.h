// Host helpers of the layer operators (layer norm, relative position bias,
// routing).  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>
#include <string>

#include "elem.h"

namespace ddp {

int32_t fail_without_context(int32_t code, const std::string& msg);   // ddp_api.hip

// What the handles of these operators have in common.
struct LayerHandle {
    int32_t device = DDP_DEVICE_NONE;
    hipStream_t stream = nullptr;
    char* mem = nullptr;                         // workspace, allocated at create
    std::string err;
};

inline int32_t layer_fail(LayerHandle* h, int32_t code, const char* msg) {
    try {
        if (h) h->err = msg;
        else return fail_without_context(code, msg);
    } catch (...) {
    }
    return code;
}

#define LAYER_HIP(h, expr)                                                                \
    do {                                                                                  \
        const hipError_t e_ = taken(expr);                                                \
        if (e_ != hipSuccess) return layer_fail((h), DDP_ERR_HIP, hipGetErrorString(e_)); \
    } while (0)

// The handle's device for the time of a call; the caller's is current again afterwards.
class OnDevice {
    int before_ = -1;

public:
    hipError_t err;
    explicit OnDevice(int device) : err(taken(hipGetDevice(&before_))) {
        if (err == hipSuccess && before_ == device) before_ = -1;
        else if (err == hipSuccess) err = taken(hipSetDevice(device));
    }
    ~OnDevice() {
        if (before_ >= 0) (void)taken(hipSetDevice(before_));
    }
    OnDevice(const OnDevice&) = delete;
    OnDevice& operator=(const OnDevice&) = delete;
};

inline bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(bytes) != 0; }
inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

inline int32_t layer_device(const char* what, int32_t device) {
    if (device < DDP_DEVICE_NONE) return layer_fail(nullptr, DDP_ERR_ARG, what);
    if (device == DDP_DEVICE_NONE) return DDP_OK;
    int count = 0;
    if (taken(hipGetDeviceCount(&count)) != hipSuccess || device >= count)
        return layer_fail(nullptr, DDP_ERR_HIP, "no such HIP device (the library needs a GPU; DDP_DEVICE_NONE checks arguments only)");
    return DDP_OK;
}

inline hipError_t layer_alloc(LayerHandle* h, int64_t bytes) {
    OnDevice on(h->device);
    return on.err != hipSuccess ? on.err : taken(hipMalloc(reinterpret_cast<void**>(&h->mem), static_cast<size_t>(bytes)));
}

// Waits for the handle's work: the caller frees what it uses.
inline void layer_release(LayerHandle* h) {
    if (h->device == DDP_DEVICE_NONE) return;
    OnDevice on(h->device);
    (void)taken(hipStreamSynchronize(h->stream));
    if (h->mem) (void)taken(hipFree(h->mem));
}

#if defined(__HIPCC__)

// The t-th tile of n in an order in which the blocks of an XCD (every eighth) have neighbouring tiles: each of the eight writes a stretch of
// memory of its own.  A grid that goes round more than once is a multiple of eight.
__device__ __forceinline__ int64_t tile_of_xcd(int64_t t, int64_t n) {
    const int64_t x = t & 7, more = n & 7;
    return x * (n >> 3) + (x < more ? x : more) + (t >> 3);
}

// Partial sums that the last block of a short launch joins, in place of another launch: stored and read with relaxed device-scope atomics, which go
// through the caches, and waited for before a block arrives (a release would write back whole caches).  Called by all threads of all
// `blocks` blocks; true in the block that arrives last, which leaves the counter at zero.
__device__ __forceinline__ void put_part(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get_part(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool arrives_last(uint32_t* counter, unsigned blocks) {
    __shared__ bool last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // this wave's parts are there
    __syncthreads();
    if (threadIdx.x == 0) {
        last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == blocks - 1;
        if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return last;
}
// The sum of `parts` parts that lie `stride` apart.
__device__ __forceinline__ double parts_sum(const float* from, int parts, int64_t stride) {
    constexpr int DEEP = 8;
    double sum = 0.0;
    for (int k = 0; k < parts; k += DEEP) {
        float x[DEEP];                               // (no condition on a load: it would be waited for before the next)
#pragma unroll
        for (int u = 0; u < DEEP; ++u) x[u] = get_part(from + min(k + u, parts - 1) * stride);
#pragma unroll
        for (int u = 0; u < DEEP; ++u) sum += k + u < parts ? x[u] : 0.0f;
    }
    return sum;
}
// A gradient of any type, added to what is there or in its place.
__device__ __forceinline__ void put_grad(char* p, int type, int64_t at, int add, double x) {
    char* to = p + at * (type == DDP_FP32 ? 4 : 2);
    if (type == DDP_FP32) store_one<DDP_FP32>(to, static_cast<float>(add ? x + load_one<DDP_FP32>(to) : x));
    else if (type == DDP_FP16) store_one<DDP_FP16>(to, static_cast<float>(add ? x + load_one<DDP_FP16>(to) : x));
    else store_one<DDP_BF16>(to, static_cast<float>(add ? x + load_one<DDP_BF16>(to) : x));
}

// Sums over the LANES (4, 8, 16, 32 or 64) neighbours of a lane, the same bits in all of them: neighbours within 16 by the VALU's lane
// moves, further ones by swaps of rows.  (A shuffle is an LDS access: six of them one after the other take some 0.4 us of a wave.)
template <int CTRL>
__device__ __forceinline__ float lane_moved(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float rows_of_16_summed(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = r[0], b = r[1];               // (a bit cast of a vector's element takes the first)
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float halves_summed(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = r[0], b = r[1];               // (a bit cast of a vector's element takes the first)
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
    x += lane_moved<0xB1>(x);                        // quad_perm: 1 0 3 2
    x += lane_moved<0x4E>(x);                        // quad_perm: 2 3 0 1
    if constexpr (LANES >= 8) x += lane_moved<0x141>(x);        // row_half_mirror
    if constexpr (LANES >= 16) x += lane_moved<0x140>(x);       // row_mirror
    if constexpr (LANES >= 32) x = rows_of_16_summed(x);
    if constexpr (LANES >= 64) x = halves_summed(x);
    return x;
}

#endif  // __HIPCC__

}  // namespace ddp
