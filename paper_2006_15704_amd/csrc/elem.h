// Element types and vector accesses shared by the optimizer and embedding
// kernels (gfx950).  Internal to the library.
//
// Tensors of callers are contiguous or rows with a stride, aligned to their
// element size and no more: a vector access may start at any element (gfx950
// executes a 16-byte access at a 2- or 4-byte aligned address as one
// instruction; an address off the 16-byte grid costs further cache lines).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "../../include/ddp_gfx950.h"

namespace ddp {

inline int elem_bytes(int dtype) { return dtype == DDP_FP32 ? 4 : 2; }
// A failure that a call reports by its status does not stay the thread's last error, which the next launch (of whoever) would report again.
inline hipError_t taken(hipError_t err) {
    if (err != hipSuccess) (void)hipGetLastError();
    return err;
}
inline bool known_dtype(int dtype) { return dtype == DDP_FP32 || dtype == DDP_FP16 || dtype == DDP_BF16; }

#if defined(__HIPCC__)

// Addresses that come from tables carry no address space; the casts keep their accesses on the global path.
#define DDP_GLOBAL_MEM __attribute__((address_space(1)))
#define DDP_CONSTANT_MEM __attribute__((address_space(4)))

template <int DT> struct ElemBytes { static constexpr int value = DT == DDP_FP32 ? 4 : 2; };
template <> struct ElemBytes<-1> { static constexpr int value = 0; };

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
template <int DWORDS, int ALIGN> struct Words;
template <> struct Words<1, 2> { typedef uint32_t type __attribute__((aligned(2))); };
template <> struct Words<1, 4> { typedef uint32_t type __attribute__((aligned(4))); };
template <> struct Words<2, 2> { typedef u32x2 type __attribute__((aligned(2))); };
template <> struct Words<2, 4> { typedef u32x2 type __attribute__((aligned(4))); };
template <> struct Words<4, 2> { typedef u32x4v type __attribute__((aligned(2))); };
template <> struct Words<4, 4> { typedef u32x4v type __attribute__((aligned(4))); };

// N consecutive elements of type DT as they lie in memory (4, 8 or 16 bytes).
template <int DT, int N> struct Raw {
    static constexpr int es = ElemBytes<DT>::value;
    static constexpr int words = N * es / 4;
    static_assert(words == 1 || words == 2 || words == 4, "one access");
    typedef typename Words<words, es>::type Mem;
    uint32_t w[words];
};

template <int DT, int N, bool NT = false>
__device__ __forceinline__ Raw<DT, N> load_raw(const void* p) {
    typedef typename Raw<DT, N>::Mem Mem;
    DDP_GLOBAL_MEM const Mem* q = (DDP_GLOBAL_MEM const Mem*)(p);
    Raw<DT, N> r;
    if constexpr (Raw<DT, N>::words == 1) {
        r.w[0] = NT ? __builtin_nontemporal_load(q) : *q;
    } else {
        const auto x = NT ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int i = 0; i < Raw<DT, N>::words; ++i) r.w[i] = x[i];
    }
    return r;
}
template <int DT, int N, bool NT = false>
__device__ __forceinline__ void store_raw(void* p, const Raw<DT, N>& r) {
    typedef typename Raw<DT, N>::Mem Mem;
    DDP_GLOBAL_MEM Mem* q = (DDP_GLOBAL_MEM Mem*)(p);
    Mem x;
    if constexpr (Raw<DT, N>::words == 1) {
        x = r.w[0];
    } else {
#pragma unroll
        for (int i = 0; i < Raw<DT, N>::words; ++i) x[i] = r.w[i];
    }
    if (NT) __builtin_nontemporal_store(x, q);
    else *q = x;
}

__device__ __forceinline__ float half_bits_to_float(uint32_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(b))); }
__device__ __forceinline__ uint32_t float_to_half_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x)); }
// round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t float_to_bf16_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

template <int DT, int N>
__device__ __forceinline__ float element(const Raw<DT, N>& r, int i) {
    if constexpr (DT == DDP_FP32) return __builtin_bit_cast(float, r.w[i]);
    const uint32_t w = r.w[i >> 1];
    if constexpr (DT == DDP_BF16) return __builtin_bit_cast(float, i & 1 ? w & 0xFFFF0000u : w << 16);
    return half_bits_to_float(i & 1 ? w >> 16 : w & 0xFFFFu);
}
// x[0..N) rounded once to DT.
template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> rounded(const float* x) {
    Raw<DT, N> r;
    if constexpr (DT == DDP_FP32) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = __builtin_bit_cast(uint32_t, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint32_t lo = DT == DDP_BF16 ? float_to_bf16_bits(x[i]) : float_to_half_bits(x[i]);
            const uint32_t hi = DT == DDP_BF16 ? float_to_bf16_bits(x[i + 1]) : float_to_half_bits(x[i + 1]);
            r.w[i >> 1] = lo | hi << 16;
        }
    }
    return r;
}

template <int DT>
__device__ __forceinline__ float load_one(const void* p) {
    if constexpr (DT == DDP_FP32) return *(DDP_GLOBAL_MEM const float*)(p);
    const uint32_t b = *(DDP_GLOBAL_MEM const uint16_t*)(p);
    if constexpr (DT == DDP_BF16) return __builtin_bit_cast(float, b << 16);
    return half_bits_to_float(b);
}
template <int DT>
__device__ __forceinline__ void store_one(void* p, float x) {
    if constexpr (DT == DDP_FP32) *(DDP_GLOBAL_MEM float*)(p) = x;
    else *(DDP_GLOBAL_MEM uint16_t*)(p) = static_cast<uint16_t>(DT == DDP_BF16 ? float_to_bf16_bits(x) : float_to_half_bits(x));
}

// N elements in as many accesses of at most 16 bytes as they take.
template <int DT, int N> struct Parts {
    static constexpr int each = N * ElemBytes<DT>::value <= 16 ? N : 16 / ElemBytes<DT>::value;
    static constexpr int count = N / each;
    Raw<DT, each> part[count];
};
template <int DT, int N, bool NT = false>
__device__ __forceinline__ Parts<DT, N> load_parts(const void* p) {
    Parts<DT, N> r;
#pragma unroll
    for (int j = 0; j < Parts<DT, N>::count; ++j)
        r.part[j] = load_raw<DT, Parts<DT, N>::each, NT>(static_cast<const char*>(p) + j * Parts<DT, N>::each * ElemBytes<DT>::value);
    return r;
}
template <int DT, int N>
__device__ __forceinline__ void widen(const Parts<DT, N>& r, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = element(r.part[i / Parts<DT, N>::each], i % Parts<DT, N>::each);
}

// The first `have` (0 to N) of N elements, zeros behind them.
template <int DT, int N, bool NT = false>
__device__ __forceinline__ void load_some(const void* p, int have, float (&x)[N]) {
    if (have >= N) {
        widen<DT, N>(load_parts<DT, N, NT>(p), x);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < have ? load_one<DT>(static_cast<const char*>(p) + i * ElemBytes<DT>::value) : 0.0f;
}
template <int DT, int N, bool NT = false>
__device__ __forceinline__ void store_some(void* p, int have, const float (&x)[N]) {
    if (have >= N) {
        constexpr int each = Parts<DT, N>::each;
#pragma unroll
        for (int j = 0; j < Parts<DT, N>::count; ++j)
            store_raw<DT, each, NT>(static_cast<char*>(p) + j * each * ElemBytes<DT>::value, rounded<DT, each>(x + j * each));
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have) store_one<DT>(static_cast<char*>(p) + i * ElemBytes<DT>::value, x[i]);
}

// Tables that no running kernel writes, read at block-uniform addresses: scalar loads.
template <typename T>
__device__ __forceinline__ T table_load(const T* p) { return *(DDP_CONSTANT_MEM const T*)(p); }

#endif  // __HIPCC__

}  // namespace ddp
