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

}  // namespace ddp
