// What follows a synchronization: the global gradient norm and the AdamW step
// over all parameter tensors at once, with the moments held in 32 bits or in 8.
//
// With g the averaged gradient, t the number of steps counting this one:
//   g' = g * grad_scale * min(1, max_norm / (|grad_scale| * norm + 1e-6))
//   m  = beta1 m + (1 - beta1) g'          v = beta2 v + (1 - beta2) g'^2
//   p  = p - lr wd p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
// Every element is read once and written once; nothing is reused, so the step
// is bound by memory and the kernels are streams of 16-byte accesses.
#include "../../include/ddp_gfx950.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "elem.h"

namespace ddp {
int32_t fail_without_context(int32_t code, const std::string& msg);   // ddp_api.hip
}

namespace {

using namespace ddp;

constexpr int kThreads = 256;
constexpr int kBlockElems = 256;                 // elements of an 8-bit state that share a scale
// A block of the step takes a tile of one tensor, `rounds` vectors of four elements a thread: one with binary32 states, two
// with 8 bits, whose tops share a division.  us, 1 / 2 / 4 rounds: 32 bits, 8 M elements 39.6 / 40.4 / 41.4, BERT-large
// 1635 / 1690 / 1688; 8 bits, 3 M 12.2 / 12.4 / 17.9, 25 M 72.3 / 68.6 / 72.1, BERT-large 932 / 910 / 889.
template <bool Q8> constexpr int kRounds = Q8 ? 2 : 1;
template <bool Q8> constexpr int kStepTile = kThreads * 4 * kRounds<Q8>;
constexpr int kNormTile = 4096;                  // elements of a tile of the norm
constexpr int kHeaderBytes = 256;                // of a state: the number of steps, then nothing
constexpr int kNormTiles = 4;                    // tiles that a block of a long norm takes
constexpr int64_t kNormLong = 90000000;          // bytes of gradients from which it is one; us, one tile a block / four (the loads of four pass
                                                 // the caches): binary32 68 MB 16.3 / 17.1, 80 MB 17.1 / 17.7, 100 MB 22.8 / 19.6,
                                                 // bfloat16 50 MB 14.1 / 15.1, 80 MB 18.9 / 20.7, 160 MB 37.9 / 30.7, 670 MB 136 / 103
                                                 // (eight: 105)
constexpr int kNormAlone = 768;                  // tiles up to which the norm is one launch; us, one / two: 500 thousand
                                                 // elements 4.9 / 6.5, 2 M 5.9 / 6.6, 3 M 6.7 / 6.5, 10 M 13.7 / 11.9
constexpr int64_t kGridBlocks = (int64_t(1) << 24) - 1; // that a grid can have: it ends at 2^32 threads
constexpr int64_t kLaunchBlocks = int64_t(1) << 20;     // of a launch of the step: a run of equal types with more tiles takes several
                                                 // (5 ms each and more, of which the drain in between is a thousandth)
constexpr int kMaskWords = 768;                  // words of the used mask that travel in one launch's arguments

struct OptSeg {                                  // 64 bytes
    uint64_t param, grad, copy;
    int64_t state;                               // first element in the states
    int64_t numel;
    int32_t step_tile0, norm_tile0;
    float lr_scale, decay_scale;
    int32_t grad_type;
    int32_t id;                                  // registration index
};
static_assert(sizeof(OptSeg) == 64, "one scalar load of sixteen words");

struct NormState {                               // in device memory
    double norm;                                 // of the registered gradients, unscaled
};
// Blocks of a running launch that are done, in kCounters groups with a cache line each, and the groups that are; 0 between launches.
// (One counter for all blocks took 10 ns a block, one after the other.)
constexpr int kCounters = 64, kCounterWords = 32, kCounterSet = (1 + kCounters) * kCounterWords;

struct StepArgs {
    const OptSeg* seg;
    const int32_t* tile_seg;
    const uint32_t* used;                        // bit i: parameter i takes part; null: all do
    const NormState* norm;                       // null: neither clipped nor looked at
    int64_t* step;
    uint32_t* counters;                          // null: another launch counts the step
    char* m;
    char* v;
    float* m_top;
    float* v_top;
    double log2_beta1, log2_beta2, lr, decay, grad_scale, max_norm;
    float beta1, rest1, beta2, rest2, eps;
    int32_t skip_nonfinite;
};

__device__ __forceinline__ OptSeg segment(const OptSeg* table, int i) {
    typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
    return __builtin_bit_cast(OptSeg, *(DDP_CONSTANT_MEM const u32x16*)(table + i));
}

// What a step does to an element that does not depend on the element.
struct Factors {
    float grad, rate, decay, root2;              // g' = g * grad; p -= decay * p + rate * m / (sqrt(v) * root2 + eps)
};

__device__ __forceinline__ Factors factors(const StepArgs& a, const OptSeg& s) {
    // 1 - beta^t in 64 bits: in 32 it would lose what beta = 0.999 leaves of it
    const double t = static_cast<double>(table_load(a.step) + 1);
    const double left1 = 1.0 - exp2(t * a.log2_beta1), left2 = 1.0 - exp2(t * a.log2_beta2);
    double g = a.grad_scale;
    if (a.max_norm > 0.0) {
        const double clip = a.max_norm / (table_load(&a.norm->norm) * fabs(a.grad_scale) + 1e-6);
        if (!(clip >= 1.0)) g *= clip;           // (a norm that is NaN shows in every parameter)
    }
    Factors f;
    f.grad = static_cast<float>(g);
    f.rate = static_cast<float>(a.lr * s.lr_scale / left1);
    f.decay = static_cast<float>(a.lr * s.lr_scale * a.decay * s.decay_scale);
    f.root2 = static_cast<float>(1.0 / sqrt(left2));
    return f;
}

// Largest of 64 lanes' values, as a scalar.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xB1, 0xF, 0xF, true)));   // quad_perm 1,0,3,2
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4E, 0xF, 0xF, true)));   // quad_perm 2,3,0,1
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x141, 0xF, 0xF, true)));  // mirror in 8
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x140, 0xF, 0xF, true)));  // mirror in 16
    const uint32_t a = max(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 0)), static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 16)));
    const uint32_t b = max(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 32)), static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 48)));
    return max(a, b);
}

// 8-bit states.  A block of 256 elements keeps its largest absolute value (binary32) and a code an element:
// first moments m = top * sign(k) (k/127)^2, second moments v = top * (k/255)^4, the nearest k in the root's scale.
// Squares and fourth powers spread the codes over 4 and 9.6 decades (what a block of gradients spans), with steps of 1.6 % at the
// top; k is at least 1 where v > 0, so that a small second moment is never taken for none and its update never blows up.
// The thresholds are (k + 1/2)^2 and ((k + 1/2)^2)^2 in binary32 (the squares are exact there), which settles the
// code whatever the last bit of an approximate root is.
constexpr float kSquare = 1.0f / (127.0f * 127.0f), kFourth = static_cast<float>(1.0 / (255.0 * 255.0 * 255.0 * 255.0));
constexpr float kSquares = 127.0f * 127.0f, kFourths = static_cast<float>(255.0 * 255.0 * 255.0 * 255.0);

__device__ __forceinline__ float first_moment(float top, int k) {
    const float x = static_cast<float>(k);
    return top * (x * fabsf(x) * kSquare);
}
__device__ __forceinline__ float second_moment(float top, uint32_t k) {
    const float x = static_cast<float>(k), y = x * x;
    return top * (y * y * kFourth);
}

// x (a whole number from 0 to 255) as byte i of `into`.
__device__ __forceinline__ uint32_t byte_of(float x, int i, uint32_t into) { return __builtin_amdgcn_cvt_pk_u8_f32(x, i, into); }

// One pass over four or five streams that are read and as many that are written.  Loads and stores carry the non-temporal hint: nothing is
// used again before everything else has been (60 M elements, binary32: 322 us without, 288 with it, 325 with it on the stores
// alone).  BERT-large, bfloat16 gradients and copies: 28 bytes an element in 1620 us, 5.8 TB/s; 8-bit states, 16 bytes, 935 us, 5.8 TB/s
// (a plain copy reaches 4.8 to 5.8).  8 bits: 75 vector instructions an element, which memory just covers; with IEEE roots and divisions
// it was 1270 us.
template <int PT, int GT, int CT, bool Q8, bool FULL>
__device__ __forceinline__ void step_tile(const StepArgs& a, const OptSeg& s, int64_t e0) {
    constexpr int PB = ElemBytes<PT>::value, GB = ElemBytes<GT>::value, CB = ElemBytes<CT>::value;
    const Factors f = factors(a, s);
    constexpr int R = kRounds<Q8>;
    float p[R][4], g[R][4], m[R][4], v[R][4], m_old[R], v_old[R];
    uint32_t m8[R], v8[R];
    const int64_t padded = (s.numel + kBlockElems - 1) / kBlockElems * kBlockElems;
    auto element_of = [&](int u) { return e0 + u * (kThreads * 4) + threadIdx.x * 4; };
    auto count_of = [&](int64_t e) { return FULL || s.numel - e >= 4 ? 4 : s.numel > e ? static_cast<int>(s.numel - e) : 0; };
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const int64_t e = element_of(u), at = s.state + e;
        const int have = count_of(e);
        const bool in_state = FULL || e < padded;
        load_some<PT, 4, true>(reinterpret_cast<const char*>(s.param) + e * PB, have, p[u]);
        load_some<GT, 4, true>(reinterpret_cast<const char*>(s.grad) + e * GB, have, g[u]);
        if constexpr (!Q8) {
            load_some<DDP_FP32, 4, true>(a.m + at * 4, in_state ? 4 : 0, m[u]);
            load_some<DDP_FP32, 4, true>(a.v + at * 4, in_state ? 4 : 0, v[u]);
        } else {
            m8[u] = in_state ? __builtin_nontemporal_load((DDP_GLOBAL_MEM const uint32_t*)(a.m + at)) : 0u;
            v8[u] = in_state ? __builtin_nontemporal_load((DDP_GLOBAL_MEM const uint32_t*)(a.v + at)) : 0u;
            m_old[u] = in_state ? *(DDP_GLOBAL_MEM const float*)(a.m_top + at / kBlockElems) : 0.0f;
            v_old[u] = in_state ? *(DDP_GLOBAL_MEM const float*)(a.v_top + at / kBlockElems) : 0.0f;
        }
    }
    uint32_t tops[2 * R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const int64_t e = element_of(u), at = s.state + e;
        const int have = count_of(e);
        uint32_t m_most = 0, v_most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (Q8) {
                m[u][i] = first_moment(m_old[u], static_cast<int8_t>(m8[u] >> (8 * i)));
                v[u][i] = second_moment(v_old[u], v8[u] >> (8 * i) & 0xFFu);
            }
            const float x = g[u][i] * f.grad;
            m[u][i] = m[u][i] * a.beta1 + x * a.rest1;
            v[u][i] = v[u][i] * a.beta2 + (x * x) * a.rest2;
            if constexpr (Q8) {                        // as integers: a NaN counts as the largest
                m_most = max(m_most, __builtin_bit_cast(uint32_t, m[u][i]) & 0x7FFFFFFFu);
                v_most = max(v_most, __builtin_bit_cast(uint32_t, v[u][i]) & 0x7FFFFFFFu);
            }
            // root and reciprocal are good to one unit in the last place, which a parameter does not show
            const float move = m[u][i] * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_sqrtf(v[u][i]), f.root2, a.eps));
            p[u][i] = p[u][i] - __builtin_fmaf(f.decay, p[u][i], f.rate * move);
        }
        store_some<PT, 4, true>(reinterpret_cast<char*>(s.param) + e * PB, have, p[u]);
        if constexpr (CT >= 0) store_some<CT, 4, true>(reinterpret_cast<char*>(s.copy) + e * CB, have, p[u]);
        if constexpr (!Q8) {
            const bool in_state = FULL || e < padded;
            store_some<DDP_FP32, 4, true>(a.m + at * 4, in_state ? 4 : 0, m[u]);
            store_some<DDP_FP32, 4, true>(a.v + at * 4, in_state ? 4 : 0, v[u]);
        } else {
            tops[2 * u] = wave_max(m_most);
            tops[2 * u + 1] = wave_max(v_most);
        }
    }
    if constexpr (Q8) {
        // The reciprocals of all the tops in one division, a lane for each.  Below the smallest normal number a block counts as
        // zeros (its reciprocal would overflow).
        uint32_t mine = 0;
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) {
            if (tops[j] < 0x00800000u) tops[j] = 0;
            if ((threadIdx.x & 63) == j) mine = tops[j];
        }
        const float inverse = mine == 0 ? 0.0f : 1.0f / __builtin_bit_cast(float, mine);
#pragma unroll
        for (int u = 0; u < R; ++u) {
            const int64_t e = element_of(u), at = s.state + e;
            const float m_inv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, inverse), 2 * u));
            const float v_inv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, inverse), 2 * u + 1));
            const float least = v_inv > 0.0f ? 1.0f : 0.0f;
            uint32_t mc = 0, vc = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // k or one less from an approximate root, then the threshold above decides (a top's q is within three roundings
                // of 127^2 or 255^4: k ends there by itself)
                float q = fabsf(m[u][i]) * m_inv * kSquares;
                float k = floorf(__builtin_amdgcn_sqrtf(q) + 0.4999f), h = k + 0.5f;
                k = h * h <= q ? k + 1.0f : k;
                mc = byte_of(copysignf(k, m[u][i]) + 128.0f, i, mc);
                q = v[u][i] * v_inv * kFourths;
                k = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(q)) + 0.4999f);
                h = (k + 0.5f) * (k + 0.5f);
                k = h * h <= q ? k + 1.0f : k;
                vc = byte_of(fmaxf(k, v[u][i] > 0.0f ? least : 0.0f), i, vc);      // (from v: q may be below the smallest number)
            }
            if (FULL || e < padded) {
                __builtin_nontemporal_store(mc ^ 0x80808080u, (DDP_GLOBAL_MEM uint32_t*)(a.m + at));
                __builtin_nontemporal_store(vc, (DDP_GLOBAL_MEM uint32_t*)(a.v + at));
                if ((threadIdx.x & 63) == 0) {
                    *(DDP_GLOBAL_MEM uint32_t*)(a.m_top + at / kBlockElems) = tops[2 * u];
                    *(DDP_GLOBAL_MEM uint32_t*)(a.v_top + at / kBlockElems) = tops[2 * u + 1];
                }
            }
        }
    }
}

__device__ __forceinline__ bool skips(const StepArgs& a) {
    return a.skip_nonfinite && !isfinite(table_load(&a.norm->norm));
}

// Called by one thread of each block: whether all other blocks have been here.  What they have stored before with device-scope
// atomics (which write through the caches) and waited for is then there to be read likewise; a release would write
// back the caches instead, which took 35 ns a block, one after the other.
__device__ __forceinline__ bool arrives_last(uint32_t* counters) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned groups = gridDim.x;                     // few blocks count themselves
    if (gridDim.x > kCounters) {
        const unsigned group = blockIdx.x % kCounters, in_group = (gridDim.x - group + kCounters - 1) / kCounters;
        uint32_t* mine = counters + (1 + group) * kCounterWords;
        if (__hip_atomic_fetch_add(mine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != in_group - 1) return false;
        __hip_atomic_store(mine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        groups = kCounters;
    }
    if (__hip_atomic_fetch_add(counters, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != groups - 1) return false;
    __hip_atomic_store(counters, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

template <int PT, int GT, int CT, bool Q8>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs a, int64_t tile_base) {
    const int64_t tile = tile_base + blockIdx.x;
    const OptSeg s = segment(a.seg, table_load(a.tile_seg + tile));
    if (skips(a)) return;
    if (a.used == nullptr || (table_load(a.used + (s.id >> 5)) >> (s.id & 31) & 1u)) {
        const int64_t e0 = (tile - s.step_tile0) * kStepTile<Q8>;
        if (e0 + kStepTile<Q8> <= s.numel) step_tile<PT, GT, CT, Q8, true>(a, s, e0);
        else step_tile<PT, GT, CT, Q8, false>(a, s, e0);
    }
    if (a.counters == nullptr) return;
    // the last block to get here counts the step: every block has read the old number by then
    __syncthreads();
    if (threadIdx.x == 0 && arrives_last(a.counters)) *a.step += 1;
}

// Counts a step whose launch has too many blocks to do it by itself, or that had none.
__global__ void count_step_kernel(StepArgs a) {
    if (!skips(a)) *a.step += 1;
}

struct MaskWords { uint32_t w[kMaskWords]; };
__global__ __launch_bounds__(kThreads) void used_mask_kernel(uint32_t* dst, MaskWords m, int words) {
    for (int i = threadIdx.x; i < words; i += kThreads) dst[i] = m.w[i];
}

// ---- the norm ----

struct NormArgs {
    const OptSeg* seg;
    const int32_t* tile_seg;
    const uint32_t* used;
    NormState* state;
    uint32_t* counters;
    double* partial;                             // one a block
    float* out;                                  // may be null
    int64_t tiles;
    double scale;                                // of what is written to out
};

template <int GT, bool NT>
__device__ __forceinline__ double tile_squares(const OptSeg& s, int64_t e0) {
    constexpr int N = GT == DDP_FP32 ? 4 : 8, GB = ElemBytes<GT>::value, rounds = kNormTile / (kThreads * N);
    float x[rounds][N];
#pragma unroll
    for (int u = 0; u < rounds; ++u) {
        const int64_t e = e0 + (u * kThreads + static_cast<int>(threadIdx.x)) * N;
        const int64_t left = s.numel - e;
        load_some<GT, N, NT>(reinterpret_cast<const char*>(s.grad) + e * GB, left >= N ? N : left > 0 ? static_cast<int>(left) : 0, x[u]);
    }
    double sum = 0.0;
#pragma unroll
    for (int u = 0; u < rounds; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double d = x[u][i];
            sum = fma(d, d, sum);
        }
    return sum;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[THREADS / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) sum += part[w];
    return sum;
}

__device__ __forceinline__ void put_norm(const NormArgs& a, double squares) {
    const double norm = sqrt(squares);
    a.state->norm = norm;
    if (a.out != nullptr) *a.out = static_cast<float>(norm * a.scale);
}

// Bound by memory: 670 MB of BERT-large's bfloat16 gradients in 103 us, 6.5 TB/s (5.6 without the non-temporal hint, which
// costs in lists that fit the 256 MB cache: 12 M elements 12.4 us without, 15.5 with it).
// Squares are summed in 64 bits: no gradient that a binary32 holds overflows or is lost.  The order of the sum (tiles by
// block, blocks by index) does not depend on which block is last.
// LAST: the block that arrives last adds the others' sums up, in place of another launch.
template <int TILES, bool LAST>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(NormArgs a) {
    double sum = 0.0;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * TILES;
#pragma unroll
    for (int k = 0; k < TILES; ++k) {
        const int64_t tile = first + k;
        if (tile >= a.tiles) break;
        const OptSeg s = segment(a.seg, table_load(a.tile_seg + tile));
        if (a.used != nullptr && !(table_load(a.used + (s.id >> 5)) >> (s.id & 31) & 1u)) continue;
        const int64_t e0 = (tile - s.norm_tile0) * kNormTile;
        if (s.grad_type == DDP_FP32) sum += tile_squares<DDP_FP32, (TILES > 1)>(s, e0);
        else if (s.grad_type == DDP_FP16) sum += tile_squares<DDP_FP16, (TILES > 1)>(s, e0);
        else sum += tile_squares<DDP_BF16, (TILES > 1)>(s, e0);
    }
    sum = block_sum<kThreads>(sum);
    if constexpr (!LAST) {
        if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
        return;
    }
    __shared__ bool last;
    if (threadIdx.x == 0) {
        __hip_atomic_store(a.partial + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = arrives_last(a.counters);
    }
    __syncthreads();
    if (!last) return;
    double total = 0.0;
    for (int i = threadIdx.x; i < static_cast<int>(gridDim.x); i += kThreads)
        total += __hip_atomic_load(a.partial + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();                                 // block_sum's words are free again
    total = block_sum<kThreads>(total);
    if (threadIdx.x == 0) put_norm(a, total);
}

__global__ __launch_bounds__(1024) void norm_join_kernel(NormArgs a, int blocks) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 8 * 1024) {
        double x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = i + k * 1024 < blocks ? a.partial[i + k * 1024] : 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k];
    }
    sum = block_sum<1024>(sum);
    if (threadIdx.x == 0) put_norm(a, sum);
}

// ---- states as values ----

// A stream: 2 bytes an element are read, 8 written, past the caches.  BERT-large, both moments: 3.4 GB in 565 us, 6.0 TB/s.
// A block takes kReadRounds vectors a thread, all on the way together, so that a cache line of scales belongs to two blocks: step and
// read-out of BERT-large with 1 / 2 / 4 / 8 of them 1467 / 1491 / 1453 / 1512 us, of 3 M elements 19.4 / 18.9 / 19.1 / 20.4.
constexpr int kReadRounds = 4;
template <bool FIRST>
__device__ __forceinline__ void read_moments(const char* codes, const float* tops, float* out, int64_t e0, int64_t elems) {
    uint32_t k[kReadRounds];
    float top[kReadRounds];
#pragma unroll
    for (int u = 0; u < kReadRounds; ++u) {
        const int64_t e = e0 + (u * kThreads + static_cast<int>(threadIdx.x)) * 4;
        k[u] = e < elems ? __builtin_nontemporal_load((DDP_GLOBAL_MEM const uint32_t*)(codes + e)) : 0u;
        top[u] = e < elems ? *(DDP_GLOBAL_MEM const float*)(tops + e / kBlockElems) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kReadRounds; ++u) {
        const int64_t e = e0 + (u * kThreads + static_cast<int>(threadIdx.x)) * 4;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FIRST) x[i] = first_moment(top[u], static_cast<int8_t>(k[u] >> (8 * i)));
            else x[i] = second_moment(top[u], k[u] >> (8 * i) & 0xFFu);
        }
        if (e < elems) store_raw<DDP_FP32, 4, true>(out + e, rounded<DDP_FP32, 4>(x));
    }
}
__global__ __launch_bounds__(kThreads) void read_state_kernel(const char* m, const char* v, const float* m_top, const float* v_top,
                                                              float* m_out, float* v_out, int64_t elems) {
    const int64_t e0 = static_cast<int64_t>(blockIdx.x) * (kThreads * 4 * kReadRounds);
    if (m_out != nullptr) read_moments<true>(m, m_top, m_out, e0, elems);
    if (v_out != nullptr) read_moments<false>(v, v_top, v_out, e0, elems);
}

// ---- host ----

struct StateLayout {
    int64_t elems = 0, m = 0, v = 0, m_top = 0, v_top = 0, bytes = 0;
};

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

StateLayout state_layout(const std::vector<int64_t>& numel, int kind) {
    StateLayout l;
    for (int64_t n : numel) l.elems += up(n, kBlockElems);
    l.m = kHeaderBytes;
    if (kind == DDP_STATE_FP32) {
        l.v = l.m + 4 * l.elems;
        l.bytes = l.v + 4 * l.elems;
        return l;
    }
    l.v = l.m + l.elems;
    l.m_top = l.v + l.elems;
    l.v_top = l.m_top + up(4 * (l.elems / kBlockElems), 256);
    l.bytes = l.v_top + up(4 * (l.elems / kBlockElems), 256);
    return l;
}

struct Launch {
    int param_type, grad_type, copy_type;
    int64_t tile_base, tiles;
};

}  // namespace

struct ddp_opt {
    int32_t device = DDP_DEVICE_NONE;
    hipStream_t stream = nullptr;
    bool registered = false, has_params = false, has_state = false, built = false, fresh_norm = false;
    std::vector<int64_t> numel;
    std::vector<int32_t> param_type, grad_type, copy_type;
    std::vector<void*> params, grads, copies;
    std::vector<float> lr_scale, decay_scale;
    int kind = DDP_STATE_FP32;
    char* state = nullptr;
    StateLayout layout;
    std::vector<Launch> launches;
    int64_t norm_tiles = 0;
    int norm_each = 1;                           // tiles that a block takes
    // device memory owned by the library: segments, tile maps, used mask, counters, partial sums, NormState
    char* mem = nullptr;
    std::vector<char*> earlier;                  // tables from before ddp_opt_set_state
    OptSeg* d_seg = nullptr;
    int32_t *d_step_seg = nullptr, *d_norm_seg = nullptr;
    uint32_t* d_used = nullptr;
    uint32_t* d_counters = nullptr;
    double* d_partial = nullptr;
    NormState* d_norm = nullptr;
    std::string err;
};

namespace {

int32_t fail(ddp_opt* o, int32_t code, const char* msg) {
    try {
        if (o) o->err = msg;
        else return ddp::fail_without_context(code, msg);
    } catch (...) {
    }
    return code;
}

#define OPT_HIP(o, expr)                                                            \
    do {                                                                            \
        const hipError_t e_ = taken(expr);                                          \
        if (e_ != hipSuccess) return fail((o), DDP_ERR_HIP, hipGetErrorString(e_)); \
    } while (0)

// C entries let no exception out; the only ones there are come from host allocations.
template <typename F>
int32_t guarded(ddp_opt* o, F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(o, DDP_ERR_HIP, "out of host memory");
    } catch (...) {
        return fail(o, DDP_ERR_HIP, "unexpected exception");
    }
}

int32_t build(ddp_opt* o) {
    const int n = static_cast<int>(o->numel.size());
    std::vector<int> order(n);
    for (int i = 0; i < n; ++i) order[i] = i;
    auto copy_of = [&](int i) { return o->copies.empty() || o->copies[i] == nullptr ? -1 : o->copy_type[i]; };
    auto group = [&](int i) { return (o->param_type[i] * 4 + o->grad_type[i]) * 4 + copy_of(i) + 1; };
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return group(a) < group(b); });
    std::vector<int64_t> first(n);
    int64_t at = 0;
    for (int i = 0; i < n; ++i) {
        first[i] = at;
        at += up(o->numel[i], kBlockElems);
    }
    const int64_t tile_elems = o->kind == DDP_STATE_8BIT ? kStepTile<true> : kStepTile<false>;
    auto tiles_of = [](int64_t numel, int64_t elems) { return (numel + elems - 1) / elems; };
    std::vector<OptSeg> seg;
    std::vector<int32_t> step_seg, norm_seg;
    o->launches.clear();
    int64_t tiles = 0, norm_tiles = 0, norm_bytes = 0;
    for (int i : order) {
        tiles += tiles_of(o->numel[i], tile_elems);
        norm_tiles += tiles_of(o->numel[i], kNormTile);
        norm_bytes += o->numel[i] * elem_bytes(o->grad_type[i]);
    }
    const int64_t read_blocks = (at + kThreads * 4 * kReadRounds - 1) / (kThreads * 4 * kReadRounds);
    if (tiles > INT32_MAX || norm_tiles > kGridBlocks * kNormTiles || read_blocks > kGridBlocks)
        return fail(o, DDP_ERR_UNSUPPORTED, "more elements than the launches of norm and read-out reach");
    step_seg.reserve(tiles);
    norm_seg.reserve(norm_tiles);
    for (int i : order) {
        if (o->numel[i] == 0) continue;
        OptSeg s{};
        s.param = o->has_params ? reinterpret_cast<uint64_t>(o->params[i]) : 0;
        s.grad = reinterpret_cast<uint64_t>(o->grads[i]);
        s.copy = copy_of(i) < 0 ? 0 : reinterpret_cast<uint64_t>(o->copies[i]);
        s.state = first[i];
        s.numel = o->numel[i];
        s.step_tile0 = static_cast<int32_t>(step_seg.size());
        s.norm_tile0 = static_cast<int32_t>(norm_seg.size());
        s.lr_scale = o->lr_scale.empty() ? 1.0f : o->lr_scale[i];
        s.decay_scale = o->decay_scale.empty() ? 1.0f : o->decay_scale[i];
        s.grad_type = o->grad_type[i];
        s.id = i;
        if (o->launches.empty() || o->launches.back().param_type != o->param_type[i] ||
            o->launches.back().grad_type != o->grad_type[i] || o->launches.back().copy_type != copy_of(i))
            o->launches.push_back(Launch{o->param_type[i], o->grad_type[i], copy_of(i), s.step_tile0, 0});
        const int64_t mine = tiles_of(s.numel, tile_elems);
        step_seg.insert(step_seg.end(), static_cast<size_t>(mine), static_cast<int32_t>(seg.size()));
        for (int64_t left = mine; left > 0;) {
            Launch& l = o->launches.back();
            const int64_t here = std::min(left, kLaunchBlocks - l.tiles);
            l.tiles += here;
            left -= here;
            if (left > 0) o->launches.push_back(Launch{l.param_type, l.grad_type, l.copy_type, l.tile_base + l.tiles, 0});
        }
        norm_seg.insert(norm_seg.end(), static_cast<size_t>(tiles_of(s.numel, kNormTile)), static_cast<int32_t>(seg.size()));
        seg.push_back(s);
    }
    OPT_HIP(o, hipSetDevice(o->device));
    if (o->mem != nullptr) {                     // built before, for the norm alone: norms under way and captured ones go on reading it
        o->earlier.push_back(o->mem);
        o->mem = nullptr;
        o->built = false;
    }
    int64_t bytes = 0;
    auto take = [&](int64_t size) {
        const int64_t at = bytes;
        bytes += up(size, 256) + 256;
        return at;
    };
    const int64_t at_seg = take(static_cast<int64_t>(seg.size() * sizeof(OptSeg))), at_step = take(tiles * 4), at_norm = take(norm_tiles * 4);
    const int64_t at_used = take((n + 31) / 32 * 4), at_counters = take(2 * kCounterSet * 4), at_state = take(sizeof(NormState));
    const int64_t at_partial = take(norm_tiles * 8);
    OPT_HIP(o, hipMalloc(reinterpret_cast<void**>(&o->mem), bytes));
    o->d_seg = reinterpret_cast<OptSeg*>(o->mem + at_seg);
    o->d_step_seg = reinterpret_cast<int32_t*>(o->mem + at_step);
    o->d_norm_seg = reinterpret_cast<int32_t*>(o->mem + at_norm);
    o->d_used = reinterpret_cast<uint32_t*>(o->mem + at_used);
    o->d_counters = reinterpret_cast<uint32_t*>(o->mem + at_counters);
    o->d_partial = reinterpret_cast<double*>(o->mem + at_partial);
    o->d_norm = reinterpret_cast<NormState*>(o->mem + at_state);
    if (!seg.empty()) {
        OPT_HIP(o, hipMemcpy(o->d_seg, seg.data(), seg.size() * sizeof(OptSeg), hipMemcpyHostToDevice));
        OPT_HIP(o, hipMemcpy(o->d_step_seg, step_seg.data(), step_seg.size() * 4, hipMemcpyHostToDevice));
        OPT_HIP(o, hipMemcpy(o->d_norm_seg, norm_seg.data(), norm_seg.size() * 4, hipMemcpyHostToDevice));
    }
    const std::vector<uint32_t> none(2 * kCounterSet);       // the step's and the norm's
    OPT_HIP(o, hipMemcpy(o->d_counters, none.data(), none.size() * 4, hipMemcpyHostToDevice));
    const NormState zero{};
    OPT_HIP(o, hipMemcpy(o->d_norm, &zero, sizeof zero, hipMemcpyHostToDevice));
    o->norm_tiles = norm_tiles;
    o->norm_each = norm_bytes < kNormLong ? 1 : kNormTiles;
    o->built = true;
    o->fresh_norm = false;
    return DDP_OK;
}

// Brings the used flags to the device; *mask is null where every parameter takes part.
int32_t upload_used(ddp_opt* o, const uint8_t* used, const uint32_t** mask) {
    *mask = nullptr;
    if (used == nullptr) return DDP_OK;
    const int n = static_cast<int>(o->numel.size());
    bool all = true;
    for (int i = 0; i < n && all; ++i) all = used[i] != 0;
    if (all) return DDP_OK;
    for (int base = 0; base < n; base += kMaskWords * 32) {
        MaskWords w{};
        const int some = std::min(n - base, kMaskWords * 32);
        for (int i = 0; i < some; ++i) w.w[i >> 5] |= static_cast<uint32_t>(used[base + i] != 0) << (i & 31);
        hipLaunchKernelGGL(used_mask_kernel, dim3(1), dim3(kThreads), 0, o->stream, o->d_used + base / 32, w, (some + 31) / 32);
        OPT_HIP(o, hipGetLastError());
    }
    *mask = o->d_used;
    return DDP_OK;
}

template <int PT, int GT, int CT>
void launch_step(const ddp_opt* o, const StepArgs& a, const Launch& l) {
    const dim3 grid(static_cast<unsigned>(l.tiles)), block(kThreads);
    if (o->kind == DDP_STATE_FP32) hipLaunchKernelGGL((adamw_kernel<PT, GT, CT, false>), grid, block, 0, o->stream, a, l.tile_base);
    else hipLaunchKernelGGL((adamw_kernel<PT, GT, CT, true>), grid, block, 0, o->stream, a, l.tile_base);
}
template <int PT, int GT>
void launch_step(const ddp_opt* o, const StepArgs& a, const Launch& l) {
    if constexpr (PT == DDP_FP32) {              // copies are of binary32 parameters
        if (l.copy_type == DDP_FP16) return launch_step<PT, GT, DDP_FP16>(o, a, l);
        if (l.copy_type == DDP_BF16) return launch_step<PT, GT, DDP_BF16>(o, a, l);
    }
    launch_step<PT, GT, -1>(o, a, l);
}
template <int PT>
void launch_step(const ddp_opt* o, const StepArgs& a, const Launch& l) {
    if (l.grad_type == DDP_FP32) launch_step<PT, DDP_FP32>(o, a, l);
    else if (l.grad_type == DDP_FP16) launch_step<PT, DDP_FP16>(o, a, l);
    else launch_step<PT, DDP_BF16>(o, a, l);
}

// Steps of up to this many blocks are counted by the launch itself; another launch takes 1 us of the GPU and 3 of the host (us
// without / with the count in the launch: 50 thousand elements 7.9 / 4.6, 1 M 8.2 / 7.1, 16 M 75.9 / 74.2).
constexpr int64_t kCountInLaunch = 16384;

bool is_finite(double x) { return std::isfinite(x); }

}  // namespace

extern "C" {

const char* ddp_opt_last_error(const ddp_opt* o) { return o ? o->err.c_str() : ddp_last_error(nullptr); }

int32_t ddp_opt_state_layout(int32_t n, const int64_t* numel, int32_t kind, int64_t* elem_offset, int64_t* where) {
    if (n <= 0 || !numel || !where) return fail(nullptr, DDP_ERR_ARG, "ddp_opt_state_layout: n <= 0 or null array");
    if (kind != DDP_STATE_FP32 && kind != DDP_STATE_8BIT) return fail(nullptr, DDP_ERR_ARG, "ddp_opt_state_layout: unknown kind of state");
    return guarded(nullptr, [&]() -> int32_t {
        int64_t at = 0;
        for (int i = 0; i < n; ++i) {
            if (numel[i] < 0) return fail(nullptr, DDP_ERR_ARG, "ddp_opt_state_layout: negative numel");
            if (elem_offset) elem_offset[i] = at;
            at += up(numel[i], kBlockElems);
        }
        const StateLayout l = state_layout(std::vector<int64_t>(numel, numel + n), kind);
        where[0] = l.m;
        where[1] = l.v;
        where[2] = l.m_top;
        where[3] = l.v_top;
        where[4] = l.elems;
        where[5] = l.bytes;
        return DDP_OK;
    });
}

int32_t ddp_opt_create(ddp_opt** out, int32_t device, void* stream) {
    if (!out) return fail(nullptr, DDP_ERR_ARG, "ddp_opt_create: out is null");
    *out = nullptr;
    if (device < DDP_DEVICE_NONE) return fail(nullptr, DDP_ERR_ARG, "ddp_opt_create: bad device");
    if (device != DDP_DEVICE_NONE) {
        int count = 0;
        if (taken(hipGetDeviceCount(&count)) != hipSuccess || device >= count)
            return fail(nullptr, DDP_ERR_HIP, "ddp_opt_create: no such HIP device (the library needs a GPU; DDP_DEVICE_NONE checks arguments only)");
    }
    ddp_opt* o = new (std::nothrow) ddp_opt();
    if (!o) return fail(nullptr, DDP_ERR_HIP, "out of host memory");
    o->device = device;
    o->stream = static_cast<hipStream_t>(stream);
    *out = o;
    return DDP_OK;
}

int32_t ddp_opt_destroy(ddp_opt* o) {
    if (!o) return DDP_ERR_ARG;
    if (o->mem || !o->earlier.empty()) {
        (void)taken(hipSetDevice(o->device));
        (void)taken(hipStreamSynchronize(o->stream));
        if (o->mem) (void)taken(hipFree(o->mem));
        for (char* mem : o->earlier) (void)taken(hipFree(mem));
    }
    delete o;
    return DDP_OK;
}

int32_t ddp_opt_register(ddp_opt* o, int32_t n, const int64_t* numel, const int32_t* param_dtype, void* const* param_ptrs,
                         const int32_t* grad_dtype, void* const* grad_ptrs) {
    if (!o) return DDP_ERR_ARG;
    if (o->registered) return fail(o, DDP_ERR_STATE, "ddp_opt_register called twice");
    if (n <= 0 || !numel || !param_dtype || !grad_dtype) return fail(o, DDP_ERR_ARG, "ddp_opt_register: n <= 0 or null array");
    const bool device = o->device != DDP_DEVICE_NONE;
    if (device && !grad_ptrs) return fail(o, DDP_ERR_ARG, "ddp_opt_register: grad_ptrs is null");
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 48)) return fail(o, DDP_ERR_ARG, "ddp_opt_register: numel out of range");
        total += numel[i];
        if (total > (int64_t(1) << 48)) return fail(o, DDP_ERR_ARG, "ddp_opt_register: numel out of range");
        if (!known_dtype(param_dtype[i]) || !known_dtype(grad_dtype[i])) return fail(o, DDP_ERR_ARG, "ddp_opt_register: unknown dtype");
        if (numel[i] == 0) continue;
        if (grad_ptrs && (!grad_ptrs[i] || reinterpret_cast<uintptr_t>(grad_ptrs[i]) % elem_bytes(grad_dtype[i])))
            return fail(o, DDP_ERR_ARG, "ddp_opt_register: gradient pointer null or not aligned to its element size");
        if (param_ptrs && (!param_ptrs[i] || reinterpret_cast<uintptr_t>(param_ptrs[i]) % elem_bytes(param_dtype[i])))
            return fail(o, DDP_ERR_ARG, "ddp_opt_register: parameter pointer null or not aligned to its element size");
    }
    return guarded(o, [&]() -> int32_t {
        std::vector<int64_t> ne(numel, numel + n);
        std::vector<int32_t> pt(param_dtype, param_dtype + n), gt(grad_dtype, grad_dtype + n);
        std::vector<void*> pp, gp;
        if (param_ptrs) pp.assign(param_ptrs, param_ptrs + n);
        if (grad_ptrs) gp.assign(grad_ptrs, grad_ptrs + n);
        o->numel.swap(ne);
        o->param_type.swap(pt);
        o->grad_type.swap(gt);
        o->params.swap(pp);
        o->grads.swap(gp);
        o->has_params = param_ptrs != nullptr || !device;
        o->registered = true;
        return o->has_params ? DDP_OK : build(o);    // with no state to come, the tables are complete
    });
}

int32_t ddp_opt_set_groups(ddp_opt* o, const float* lr_scale, const float* decay_scale) {
    if (!o) return DDP_ERR_ARG;
    if (!o->registered) return fail(o, DDP_ERR_STATE, "ddp_opt_set_groups before ddp_opt_register");
    if (o->has_state) return fail(o, DDP_ERR_STATE, "ddp_opt_set_groups after ddp_opt_set_state");
    const size_t n = o->numel.size();
    for (size_t i = 0; i < n; ++i)
        if ((lr_scale && !is_finite(lr_scale[i])) || (decay_scale && !is_finite(decay_scale[i])))
            return fail(o, DDP_ERR_ARG, "ddp_opt_set_groups: a factor is not finite");
    return guarded(o, [&]() -> int32_t {
        std::vector<float> lr, decay;
        if (lr_scale) lr.assign(lr_scale, lr_scale + n);
        if (decay_scale) decay.assign(decay_scale, decay_scale + n);
        o->lr_scale.swap(lr);
        o->decay_scale.swap(decay);
        return DDP_OK;
    });
}

int32_t ddp_opt_set_copies(ddp_opt* o, const int32_t* copy_dtype, void* const* copy_ptrs) {
    if (!o) return DDP_ERR_ARG;
    if (!o->registered) return fail(o, DDP_ERR_STATE, "ddp_opt_set_copies before ddp_opt_register");
    if (o->has_state) return fail(o, DDP_ERR_STATE, "ddp_opt_set_copies after ddp_opt_set_state");
    if (!copy_dtype || !copy_ptrs) return fail(o, DDP_ERR_ARG, "ddp_opt_set_copies: null array");
    const size_t n = o->numel.size();
    for (size_t i = 0; i < n; ++i) {
        if (!copy_ptrs[i]) continue;
        if (copy_dtype[i] != DDP_FP16 && copy_dtype[i] != DDP_BF16) return fail(o, DDP_ERR_ARG, "ddp_opt_set_copies: copies are fp16 or bf16");
        if (o->param_type[i] != DDP_FP32) return fail(o, DDP_ERR_ARG, "ddp_opt_set_copies: copies are of binary32 parameters");
        if (reinterpret_cast<uintptr_t>(copy_ptrs[i]) % 2) return fail(o, DDP_ERR_ARG, "ddp_opt_set_copies: copy pointer not aligned to its element size");
    }
    return guarded(o, [&]() -> int32_t {
        std::vector<int32_t> ct(copy_dtype, copy_dtype + n);
        std::vector<void*> cp(copy_ptrs, copy_ptrs + n);
        o->copy_type.swap(ct);
        o->copies.swap(cp);
        return DDP_OK;
    });
}

int32_t ddp_opt_set_state(ddp_opt* o, int32_t kind, void* state, int64_t bytes) {
    if (!o) return DDP_ERR_ARG;
    if (!o->registered) return fail(o, DDP_ERR_STATE, "ddp_opt_set_state before ddp_opt_register");
    if (o->has_state) return fail(o, DDP_ERR_STATE, "ddp_opt_set_state called twice");
    if (kind != DDP_STATE_FP32 && kind != DDP_STATE_8BIT) return fail(o, DDP_ERR_ARG, "ddp_opt_set_state: unknown kind of state");
    if (!o->has_params) return fail(o, DDP_ERR_STATE, "ddp_opt_set_state: no parameters are registered");
    return guarded(o, [&]() -> int32_t {
        const StateLayout l = state_layout(o->numel, kind);
        if (bytes < l.bytes) return fail(o, DDP_ERR_ARG, "ddp_opt_set_state: fewer bytes than ddp_opt_state_layout asks for");
        if (o->device != DDP_DEVICE_NONE && !state) return fail(o, DDP_ERR_ARG, "ddp_opt_set_state: state is null");
        if (reinterpret_cast<uintptr_t>(state) % 16) return fail(o, DDP_ERR_ARG, "ddp_opt_set_state: state not aligned to 16 bytes");
        o->kind = kind;
        o->state = static_cast<char*>(state);
        o->layout = l;
        if (o->device != DDP_DEVICE_NONE) {
            const int32_t rc = build(o);
            if (rc != DDP_OK) return rc;
        }
        o->has_state = true;
        return DDP_OK;
    });
}

int32_t ddp_opt_grad_norm(ddp_opt* o, double grad_scale, const uint8_t* used, float* norm_out) {
    if (!o) return DDP_ERR_ARG;
    if (!o->registered) return fail(o, DDP_ERR_STATE, "ddp_opt_grad_norm before ddp_opt_register");
    if (!is_finite(grad_scale)) return fail(o, DDP_ERR_ARG, "ddp_opt_grad_norm: grad_scale is not finite");
    if (reinterpret_cast<uintptr_t>(norm_out) % 4) return fail(o, DDP_ERR_ARG, "ddp_opt_grad_norm: norm_out not aligned to 4 bytes");
    if (o->device == DDP_DEVICE_NONE) return fail(o, DDP_ERR_NO_DEVICE, "ddp_opt_grad_norm without a device");
    return guarded(o, [&]() -> int32_t {
        if (!o->built) {
            const int32_t rc = build(o);
            if (rc != DDP_OK) return rc;
        }
        OPT_HIP(o, hipSetDevice(o->device));
        NormArgs a{};
        const int32_t rc = upload_used(o, used, &a.used);
        if (rc != DDP_OK) return rc;
        a.seg = o->d_seg;
        a.tile_seg = o->d_norm_seg;
        a.state = o->d_norm;
        a.counters = o->d_counters + kCounterSet;
        a.partial = o->d_partial;
        a.out = norm_out;
        a.tiles = o->norm_tiles;
        a.scale = std::fabs(grad_scale);
        if (o->norm_tiles <= kNormAlone) {
            hipLaunchKernelGGL((grad_norm_kernel<1, true>), dim3(std::max(1, static_cast<int>(o->norm_tiles))), dim3(kThreads), 0, o->stream, a);
        } else {
            const int blocks = static_cast<int>((o->norm_tiles + o->norm_each - 1) / o->norm_each);
            if (o->norm_each == 1) hipLaunchKernelGGL((grad_norm_kernel<1, false>), dim3(blocks), dim3(kThreads), 0, o->stream, a);
            else hipLaunchKernelGGL((grad_norm_kernel<kNormTiles, false>), dim3(blocks), dim3(kThreads), 0, o->stream, a);
            OPT_HIP(o, hipGetLastError());
            hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(1024), 0, o->stream, a, blocks);
        }
        OPT_HIP(o, hipGetLastError());
        o->fresh_norm = true;
        return DDP_OK;
    });
}

int32_t ddp_opt_adamw_step(ddp_opt* o, double lr, double beta1, double beta2, double eps, double weight_decay,
                           double grad_scale, double max_norm, int32_t skip_nonfinite, const uint8_t* used) {
    if (!o) return DDP_ERR_ARG;
    if (!o->has_state) return fail(o, DDP_ERR_STATE, "ddp_opt_adamw_step before ddp_opt_set_state");
    if (!is_finite(lr) || !is_finite(weight_decay) || !is_finite(grad_scale) || !is_finite(max_norm) || !is_finite(eps) || eps < 0.0)
        return fail(o, DDP_ERR_ARG, "ddp_opt_adamw_step: an argument is not finite, or eps is negative");
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return fail(o, DDP_ERR_ARG, "ddp_opt_adamw_step: betas outside [0, 1)");
    if (o->device == DDP_DEVICE_NONE) return fail(o, DDP_ERR_NO_DEVICE, "ddp_opt_adamw_step without a device");
    if ((max_norm > 0.0 || skip_nonfinite) && !o->fresh_norm)
        return fail(o, DDP_ERR_STATE, "ddp_opt_adamw_step: clipping and skipping need ddp_opt_grad_norm since the last step");
    return guarded(o, [&]() -> int32_t {
        OPT_HIP(o, hipSetDevice(o->device));
        StepArgs a{};
        const int32_t rc = upload_used(o, used, &a.used);
        if (rc != DDP_OK) return rc;
        a.seg = o->d_seg;
        a.tile_seg = o->d_step_seg;
        a.norm = o->d_norm;
        a.step = reinterpret_cast<int64_t*>(o->state);
        a.m = o->state + o->layout.m;
        a.v = o->state + o->layout.v;
        a.m_top = reinterpret_cast<float*>(o->state + o->layout.m_top);
        a.v_top = reinterpret_cast<float*>(o->state + o->layout.v_top);
        a.log2_beta1 = std::log2(beta1);
        a.log2_beta2 = std::log2(beta2);
        a.lr = lr;
        a.decay = weight_decay;
        a.grad_scale = grad_scale;
        a.max_norm = max_norm;
        a.beta1 = static_cast<float>(beta1);
        a.rest1 = static_cast<float>(1.0 - beta1);
        a.beta2 = static_cast<float>(beta2);
        a.rest2 = static_cast<float>(1.0 - beta2);
        // below the smallest normal number the reciprocal takes eps for 0: an element of no gradient would be 0 / 0, not 0 / eps
        a.eps = eps > 0.0 ? std::max(static_cast<float>(eps), FLT_MIN) : 0.0f;
        a.skip_nonfinite = skip_nonfinite != 0;
        bool counted = false;
        for (size_t i = 0; i < o->launches.size(); ++i) {
            const Launch& l = o->launches[i];
            counted = i + 1 == o->launches.size() && l.tiles <= kCountInLaunch;
            a.counters = counted ? o->d_counters : nullptr;
            if (l.param_type == DDP_FP32) launch_step<DDP_FP32>(o, a, l);
            else if (l.param_type == DDP_FP16) launch_step<DDP_FP16>(o, a, l);
            else launch_step<DDP_BF16>(o, a, l);
            OPT_HIP(o, hipGetLastError());
        }
        if (!counted) {
            hipLaunchKernelGGL(count_step_kernel, dim3(1), dim3(1), 0, o->stream, a);
            OPT_HIP(o, hipGetLastError());
        }
        o->fresh_norm = false;
        return DDP_OK;
    });
}

int32_t ddp_opt_read_state(ddp_opt* o, float* m_out, float* v_out) {
    if (!o) return DDP_ERR_ARG;
    if (!o->has_state) return fail(o, DDP_ERR_STATE, "ddp_opt_read_state before ddp_opt_set_state");
    if (o->kind != DDP_STATE_8BIT) return fail(o, DDP_ERR_STATE, "ddp_opt_read_state: 32-bit states are the values themselves");
    if (reinterpret_cast<uintptr_t>(m_out) % 4 || reinterpret_cast<uintptr_t>(v_out) % 4)
        return fail(o, DDP_ERR_ARG, "ddp_opt_read_state: output not aligned to 4 bytes");
    if (o->device == DDP_DEVICE_NONE) return fail(o, DDP_ERR_NO_DEVICE, "ddp_opt_read_state without a device");
    if ((!m_out && !v_out) || o->layout.elems == 0) return DDP_OK;
    return guarded(o, [&]() -> int32_t {
        OPT_HIP(o, hipSetDevice(o->device));
        const int64_t blocks = (o->layout.elems + kThreads * 4 * kReadRounds - 1) / (kThreads * 4 * kReadRounds);
        hipLaunchKernelGGL(read_state_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, o->stream,
                           o->state + o->layout.m, o->state + o->layout.v, reinterpret_cast<const float*>(o->state + o->layout.m_top),
                           reinterpret_cast<const float*>(o->state + o->layout.v_top), m_out, v_out, o->layout.elems);
        OPT_HIP(o, hipGetLastError());
        return DDP_OK;
    });
}

}  // extern "C"
