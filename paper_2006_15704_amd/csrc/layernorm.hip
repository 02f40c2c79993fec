// Layer norm over the last dimension with the residual sum in front of it, and its gradients.
//
//   s = x (+ residual),  xh = (s - mean) rstd,  y = xh gamma + beta
//   g = dy gamma,  dx = (g - mean(g) - xh mean(g xh)) rstd (+ dsum)
//   dgamma = sum over the rows of dy xh,  dbeta = sum over the rows of dy
//
// Bound by memory: some 8 operations an element forward, 14 backward.  16384 x 1024 bfloat16 with a residual (134 MB) takes 20.9 us, 6.4 TB/s;
// backward 32768 x 4096 bfloat16 with dsum (1074 MB) 195 us, 5.5 TB/s, 5 of them the join of the parameters' sums; 20011 x 771 binary32 (155 MB)
// 35 us, 28 and 5 with what lies between them.
#include "layer_host.h"

struct ddp_layernorm : ddp::LayerHandle {
    int64_t width = 0;
    int32_t chunks = 0;                          // row chunks that the workspace holds sums of
    float* partial = nullptr;                    // [chunks][2][width]
    uint32_t* counter = nullptr;
};

namespace {

using namespace ddp;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int64_t kMaxWidth = int64_t(1) << 20, kMaxRows = INT32_MAX;
// Results of this size and more are stored past the caches, where their reader would not find them any more (16384 x 1024 with a residual 21.1 us
// against 26.3, backward 20011 x 771 34.9 against 38.7; one row of 1024 the other way 4.9 against 5.9).
constexpr int64_t kStreamBytes = int64_t(4) << 20;

struct ForwardArgs {
    const char *x, *residual, *gamma, *beta;
    char *sum, *y;
    float *mean, *rstd;
    int64_t rows, x_stride, residual_stride, sum_stride, y_stride;
    int32_t width, param, stream;
    float eps;
};
struct BackwardArgs {
    const char *dy, *x, *gamma, *dsum;
    const float *mean, *rstd;
    char *dx;
    float* partial;
    uint32_t* counter;                               // of the blocks that have arrived, where the last one joins
    char *dgamma, *dbeta;
    int64_t rows, dy_stride, x_stride, dsum_stride, dx_stride, rows_per_chunk;
    int32_t width, param, chunks, stream, grad, add;
};

// gamma or beta: `none` where there is none.
template <int N>
__device__ __forceinline__ void load_param(const char* p, int type, int64_t at, int have, float none, float (&v)[N]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = none;
    } else if (type == DDP_FP32) {
        load_some<DDP_FP32, N>(p + at * 4, have, v);
    } else if (type == DDP_FP16) {
        load_some<DDP_FP16, N>(p + at * 2, have, v);
    } else {
        load_some<DDP_BF16, N>(p + at * 2, have, v);
    }
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// Of all threads of a block, in all of them.
__device__ __forceinline__ float block_sum(float x, float* part) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float sum = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += part[w];
    return sum;
}

// ---- rows that fit into the registers of a team ----
//
// A team is LANES neighbouring lanes or WAVES waves with EACH elements a lane: a row is read once (three passes, the later ones from the caches,
// took 54 us where this takes 21), in whole 16-byte vectors that are all on
// the way together, and its sums are taken in registers.  Vector v of lane l is at column (v lanes + l) N; the one that would reach over the
// end of the row is moved back to end with it, and what it shares with the vector in front of it counts there.
constexpr int kMostEach = 16;

template <int XT, int YT, int LANES_, int WAVES_, int THREADS_, int EACH_>
struct Team {
    static constexpr int LANES = LANES_, WAVES = WAVES_, THREADS = THREADS_, EACH = EACH_;
    static constexpr int N = XT == DDP_FP32 ? 4 : 8, V = EACH / N, SIZE = LANES * WAVES, TEAMS = THREADS / SIZE;
    static_assert(LANES == 64 || WAVES == 1, "a team of several waves has whole ones");
    int at[V], own[V];                               // own: elements from here on are the vector's; N: nothing here
    bool ragged;

    __host__ __device__ __forceinline__ explicit Team(int width) {
#if defined(__HIP_DEVICE_COMPILE__)
        const int lane = static_cast<int>(threadIdx.x) % SIZE;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * SIZE + lane) * N;
            at[v] = c + N <= width ? c : width - N;
            own[v] = c >= width ? N : c - at[v];
        }
        ragged = width != SIZE * EACH;
#endif
    }
    // The block's team that a thread belongs to; where that is a wave's, its rows' addresses are scalars.
    __device__ __forceinline__ static int mine() {
        const int team = static_cast<int>(threadIdx.x) / SIZE;
        return LANES == 64 ? __builtin_amdgcn_readfirstlane(team) : team;
    }
    // Elements that are another vector's, or of no row, as zeros.
    __device__ __forceinline__ void clear_shared(bool live, float (&x)[V][N]) const {
        if (!ragged && live) return;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) x[v][i] = live && i >= own[v] ? x[v][i] : 0.0f;
    }
    // (No condition, or each load would be waited for before the next: a vector that has nothing reads the row's end.)
    template <int DT>
    __device__ __forceinline__ void load(const char* row, Parts<DT, N> (&raw)[V]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = load_parts<DT, N>(row + static_cast<unsigned>(at[v]) * ElemBytes<DT>::value);
    }
    template <int DT, bool NT = false>
    __device__ __forceinline__ void store(char* row, bool live, const float (&x)[V][N]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live || own[v] == N) continue;
            char* to = row + static_cast<unsigned>(at[v]) * ElemBytes<DT>::value;
            if (own[v] == 0) {
                store_some<DT, N, NT>(to, N, x[v]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i >= own[v]) store_one<DT>(to + i * ElemBytes<DT>::value, x[v][i]);
            }
        }
    }
    __device__ __forceinline__ void params(const char* p, int type, float none, float (&x)[V][N]) const {
#pragma unroll
        for (int v = 0; v < V; ++v) load_param<N>(p, type, at[v], N, none, x[v]);
    }
    // Sums over the team.  Several waves meet in LDS: `meet` has room for two values of each wave, and alternates.
    __device__ __forceinline__ void sum(float& a, float* meet) const {
        a = lanes_sum<LANES>(a);
        if constexpr (WAVES > 1) {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) meet[wave] = a;
            __syncthreads();
            const float* mine = meet + wave / WAVES * WAVES;
            a = mine[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) a += mine[w];
        }
    }
    __device__ __forceinline__ void sum(float& a, float& b, float* meet) const {
        a = lanes_sum<LANES>(a);
        b = lanes_sum<LANES>(b);
        if constexpr (WAVES > 1) {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
                meet[wave * 2] = a;
                meet[wave * 2 + 1] = b;
            }
            __syncthreads();
            const float* mine = meet + wave / WAVES * WAVES * 2;
            a = mine[0];
            b = mine[1];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) {
                a += mine[w * 2];
                b += mine[w * 2 + 1];
            }
        }
    }
};

template <typename T, int DT>
__device__ __forceinline__ void put(const T& team, int stream, char* row, bool live, const float (&x)[T::V][T::N]) {
    if (stream) team.template store<DT, true>(row, live, x);
    else team.template store<DT>(row, live, x);
}

template <int XT, int YT, typename T>
__global__ __launch_bounds__(T::THREADS) void forward_team_kernel(ForwardArgs a) {
    constexpr int N = T::N, V = T::V;
    __shared__ float meet[2][T::THREADS / 64];
    const T team(a.width);
    float gamma[V][N], beta[V][N];
    team.params(a.gamma, a.param, 1.0f, gamma);
    team.params(a.beta, a.param, 0.0f, beta);
    const float each = 1.0f / a.width;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * T::TEAMS; base < a.rows; base += static_cast<int64_t>(gridDim.x) * T::TEAMS) {
        const int64_t row = base + T::mine();
        const bool live = row < a.rows;
        const int64_t from = live ? row : a.rows - 1;
        Parts<XT, N> x[V], r[V];
        team.template load<XT>(a.x + from * a.x_stride * ElemBytes<XT>::value, x);
        if (a.residual != nullptr) team.template load<XT>(a.residual + from * a.residual_stride * ElemBytes<XT>::value, r);
        float s[V][N], sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) widen<XT, N>(x[v], s[v]);
        if (a.residual != nullptr) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float more[N];
                widen<XT, N>(r[v], more);
#pragma unroll
                for (int i = 0; i < N; ++i) s[v][i] += more[i];
            }
        }
        if (a.sum != nullptr) put<T, XT>(team, a.stream, a.sum + row * a.sum_stride * ElemBytes<XT>::value, live, s);
        team.clear_shared(live, s);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) sum += s[v][i];
        team.sum(sum, meet[0]);
        const float mean = sum * each;
        float squares = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) s[v][i] -= mean;
        team.clear_shared(live, s);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) squares += s[v][i] * s[v][i];
        team.sum(squares, meet[1]);
        const float rstd = 1.0f / sqrtf(squares * each + a.eps);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) s[v][i] = s[v][i] * rstd * gamma[v][i] + beta[v][i];
        put<T, YT>(team, a.stream, a.y + row * a.y_stride * ElemBytes<YT>::value, live, s);
        if (live && threadIdx.x % T::SIZE == 0) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
    }
}

// One pass for all three gradients.  The block's teams sum dgamma and dbeta over their rows in binary32, meet in LDS by halves, and leave one row
// of sums for the join, which adds those in binary64: no atomics, the same order in every call.
template <int XT, int YT, typename T>
__global__ __launch_bounds__(T::THREADS) void backward_team_kernel(BackwardArgs a) {
    constexpr int N = T::N, V = T::V;
    constexpr bool WIDE = T::LANES == 64;            // narrower teams meet within their wave first
    constexpr int MEET = WIDE ? T::TEAMS : T::THREADS / 64;
    __shared__ float meet[2][T::THREADS / 64 * 2];
    __shared__ float part[MEET > 1 ? MEET / 2 : 1][2][MEET > 1 ? T::SIZE * T::EACH : 1];
    const T team(a.width);
    // of the widest rows a lane's sums of the parameters' gradients are in LDS, which registers do not suffice for
    constexpr bool IN_LDS = T::WAVES == 16 && T::EACH == kMostEach;
    __shared__ __attribute__((aligned(16))) float held[IN_LDS ? 2 * V : 1][IN_LDS ? T::SIZE : 1][N];
    float gamma[V][N], dgamma[V][N] = {}, dbeta[V][N] = {};
    team.params(a.gamma, a.param, 1.0f, gamma);
    auto hold = [&](int at, float (&x)[N], bool add) {
#pragma unroll
        for (int i = 0; i < N; ++i) held[at][threadIdx.x][i] = add ? held[at][threadIdx.x][i] + x[i] : x[i];
    };
    if constexpr (IN_LDS) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            hold(v, dgamma[v], false);
            hold(V + v, dbeta[v], false);
        }
    }
    const float each = 1.0f / a.width;
    int turn = 0;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * T::TEAMS; base < a.rows; base += static_cast<int64_t>(gridDim.x) * T::TEAMS) {
        const int64_t row = base + T::mine();
        const bool live = row < a.rows;
        const int64_t from = live ? row : a.rows - 1;
        Parts<XT, N> x[V], more[V];
        Parts<YT, N> dy[V];
        team.template load<YT>(a.dy + from * a.dy_stride * ElemBytes<YT>::value, dy);
        team.template load<XT>(a.x + from * a.x_stride * ElemBytes<XT>::value, x);
        if (a.dsum != nullptr && a.dx != nullptr) team.template load<XT>(a.dsum + from * a.dsum_stride * ElemBytes<XT>::value, more);
        const float mean = a.mean[from], rstd = a.rstd[from];
        float g[V][N], xh[V][N], of_g = 0.0f, of_gx = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            widen<YT, N>(dy[v], g[v]);
            widen<XT, N>(x[v], xh[v]);
#pragma unroll
            for (int i = 0; i < N; ++i) xh[v][i] = (xh[v][i] - mean) * rstd;
        }
        team.clear_shared(live, g);
        team.clear_shared(live, xh);
        if constexpr (IN_LDS) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = g[v][i] * xh[v][i];
                hold(v, x, true);
                hold(V + v, g[v], true);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dgamma[v][i] += g[v][i] * xh[v][i];
                    dbeta[v][i] += g[v][i];
                }
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                g[v][i] *= gamma[v][i];
                of_g += g[v][i];
                of_gx += g[v][i] * xh[v][i];
            }
        if (a.dx == nullptr) continue;
        team.sum(of_g, of_gx, meet[turn]);
        turn ^= 1;
        const float c1 = of_g * each, c2 = of_gx * each;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) g[v][i] = (g[v][i] - c1 - xh[v][i] * c2) * rstd;
        if (a.dsum != nullptr) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float m[N];
                widen<XT, N>(more[v], m);
#pragma unroll
                for (int i = 0; i < N; ++i) g[v][i] += m[i];
            }
        }
        put<T, XT>(team, a.stream, a.dx + row * a.dx_stride * ElemBytes<XT>::value, live, g);
    }
    if (a.partial == nullptr) return;
    if constexpr (IN_LDS) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                dgamma[v][i] = held[v][threadIdx.x][i];
                dbeta[v][i] = held[V + v][threadIdx.x][i];
            }
    }
    if constexpr (!WIDE) {
#pragma unroll
        for (int d = T::LANES; d < 64; d <<= 1)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dgamma[v][i] += __shfl_xor(dgamma[v][i], d);
                    dbeta[v][i] += __shfl_xor(dbeta[v][i], d);
                }
    }
    const int me = WIDE ? threadIdx.x / T::SIZE : threadIdx.x >> 6, lane = threadIdx.x % T::SIZE;
#pragma unroll
    for (int half = MEET / 2; half > 0; half >>= 1) {
        if (me >= half && me < 2 * half) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    part[me - half][0][(v * N + i) * T::SIZE + lane] = dgamma[v][i];
                    part[me - half][1][(v * N + i) * T::SIZE + lane] = dbeta[v][i];
                }
        }
        __syncthreads();
        if (me < half) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dgamma[v][i] += part[me][0][(v * N + i) * T::SIZE + lane];
                    dbeta[v][i] += part[me][1][(v * N + i) * T::SIZE + lane];
                }
        }
        __syncthreads();
    }
    float* to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.width;
    if (a.counter == nullptr) {
        if (threadIdx.x >= T::SIZE) return;
        team.template store<DDP_FP32>(reinterpret_cast<char*>(to), true, dgamma);
        team.template store<DDP_FP32>(reinterpret_cast<char*>(to + a.width), true, dbeta);
        return;
    }
    if (threadIdx.x < T::SIZE) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i >= team.own[v]) {
                    put_part(to + team.at[v] + i, dgamma[v][i]);
                    put_part(to + a.width + team.at[v] + i, dbeta[v][i]);
                }
    }
    if (!arrives_last(a.counter, gridDim.x)) return;
    for (int c = threadIdx.x; c < 2 * a.width; c += T::THREADS) {
        char* grad = c < a.width ? a.dgamma : a.dbeta;
        if (grad != nullptr) put_grad(grad, a.grad, c < a.width ? c : c - a.width, a.add, parts_sum(a.partial + c, gridDim.x, 2 * static_cast<int64_t>(a.width)));
    }
}

// ---- other rows ----

// A block a row, three passes over it (the second and third come from the caches): rows shorter than a vector or longer than 16384 elements
// (2048 x 20000: 162 us forward, 157 backward, 2 TB/s).
constexpr int kN = 4;
template <int XT>
__device__ __forceinline__ void load_sum(const ForwardArgs& a, int64_t row, int c, float (&s)[kN]) {
    const int have = a.width - c;
    load_some<XT, kN>(a.x + (row * a.x_stride + c) * ElemBytes<XT>::value, have, s);
    if (a.residual != nullptr) {
        float r[kN];
        load_some<XT, kN>(a.residual + (row * a.residual_stride + c) * ElemBytes<XT>::value, have, r);
#pragma unroll
        for (int i = 0; i < kN; ++i) s[i] += r[i];
    }
}
template <int XT, int YT>
__global__ __launch_bounds__(kThreads) void forward_kernel(ForwardArgs a) {
    __shared__ float part[kWaves];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f;
        for (int c = threadIdx.x * kN; c < a.width; c += kThreads * kN) {
            float s[kN];
            load_sum<XT>(a, row, c, s);
#pragma unroll
            for (int i = 0; i < kN; ++i) sum += s[i];
        }
        const float mean = block_sum(sum, part) / a.width;
        float squares = 0.0f;
        for (int c = threadIdx.x * kN; c < a.width; c += kThreads * kN) {
            float s[kN];
            load_sum<XT>(a, row, c, s);
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (c + i < a.width) squares += (s[i] - mean) * (s[i] - mean);
        }
        const float rstd = 1.0f / sqrtf(block_sum(squares, part) / a.width + a.eps);
        for (int c = threadIdx.x * kN; c < a.width; c += kThreads * kN) {
            const int have = a.width - c;
            float s[kN], g[kN], b[kN];
            load_sum<XT>(a, row, c, s);
            load_param<kN>(a.gamma, a.param, c, have, 1.0f, g);
            load_param<kN>(a.beta, a.param, c, have, 0.0f, b);
            if (a.sum != nullptr) store_some<XT, kN>(a.sum + (row * a.sum_stride + c) * ElemBytes<XT>::value, have, s);
#pragma unroll
            for (int i = 0; i < kN; ++i) s[i] = (s[i] - mean) * rstd * g[i] + b[i];
            store_some<YT, kN>(a.y + (row * a.y_stride + c) * ElemBytes<YT>::value, have, s);
        }
        if (threadIdx.x == 0) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
    }
}

template <int XT, int YT>
__device__ __forceinline__ void load_pair(const BackwardArgs& a, int64_t row, int c, float mean, float rstd, float (&dy)[kN], float (&xh)[kN]) {
    const int have = a.width - c;
    load_some<YT, kN>(a.dy + (row * a.dy_stride + c) * ElemBytes<YT>::value, have, dy);
    load_some<XT, kN>(a.x + (row * a.x_stride + c) * ElemBytes<XT>::value, have, xh);
#pragma unroll
    for (int i = 0; i < kN; ++i) xh[i] = (xh[i] - mean) * rstd;
}
template <int XT, int YT>
__global__ __launch_bounds__(kThreads) void backward_rows_kernel(BackwardArgs a) {
    __shared__ float part[kWaves];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float of_g = 0.0f, of_gx = 0.0f;
        for (int c = threadIdx.x * kN; c < a.width; c += kThreads * kN) {
            float dy[kN], xh[kN], gamma[kN];
            load_pair<XT, YT>(a, row, c, mean, rstd, dy, xh);
            load_param<kN>(a.gamma, a.param, c, a.width - c, 1.0f, gamma);
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                if (c + i >= a.width) continue;
                of_g += dy[i] * gamma[i];
                of_gx += dy[i] * gamma[i] * xh[i];
            }
        }
        const float c1 = block_sum(of_g, part) / a.width, c2 = block_sum(of_gx, part) / a.width;
        for (int c = threadIdx.x * kN; c < a.width; c += kThreads * kN) {
            const int have = a.width - c;
            float dy[kN], xh[kN], gamma[kN], more[kN] = {};
            load_pair<XT, YT>(a, row, c, mean, rstd, dy, xh);
            load_param<kN>(a.gamma, a.param, c, have, 1.0f, gamma);
            if (a.dsum != nullptr) load_some<XT, kN>(a.dsum + (row * a.dsum_stride + c) * ElemBytes<XT>::value, have, more);
#pragma unroll
            for (int i = 0; i < kN; ++i) dy[i] = (dy[i] * gamma[i] - c1 - xh[i] * c2) * rstd + more[i];
            store_some<XT, kN>(a.dx + (row * a.dx_stride + c) * ElemBytes<XT>::value, have, dy);
        }
    }
}

// A block has 64 kN columns and a chunk of the rows, which go round its waves.
template <int XT, int YT>
__global__ __launch_bounds__(kThreads) void backward_columns_kernel(BackwardArgs a) {
    __shared__ float part[kWaves][2][64 * kN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (blockIdx.x * 64 + lane) * kN;
    const int64_t from = blockIdx.y * a.rows_per_chunk, to = min(from + a.rows_per_chunk, a.rows);
    float dgamma[kN] = {}, dbeta[kN] = {};
    if (c < a.width) {
        for (int64_t row = from + wave; row < to; row += kWaves) {
            float dy[kN], xh[kN];
            load_pair<XT, YT>(a, row, c, a.mean[row], a.rstd[row], dy, xh);
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                dgamma[i] += dy[i] * xh[i];
                dbeta[i] += dy[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        part[wave][0][i * 64 + lane] = dgamma[i];
        part[wave][1][i * 64 + lane] = dbeta[i];
    }
    __syncthreads();
    if (wave >= 2 || c >= a.width) return;           // wave 0 has dgamma, wave 1 dbeta
    float* to_part = a.partial + (static_cast<int64_t>(blockIdx.y) * 2 + wave) * a.width;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += part[w][wave][i * 64 + lane];
        if (c + i < a.width) to_part[c + i] = sum;
    }
}

struct JoinArgs {
    const float* partial;
    char *dgamma, *dbeta;
    int32_t width, chunks, grad, add;
};
// blockIdx.y: dgamma, dbeta.  A wave has 64 columns of a share of the chunks, kJoinWaves of them meet in LDS.
constexpr int kJoinWaves = 16, kJoinDeep = 16;
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(JoinArgs a) {
    __shared__ double part[kJoinWaves][64];
    char* out = blockIdx.y == 0 ? a.dgamma : a.dbeta;
    if (out == nullptr) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    double sum = 0.0;
    if (c < a.width) {
        const float* from = a.partial + static_cast<int64_t>(blockIdx.y) * a.width + c;
        for (int k = wave; k < a.chunks; k += kJoinWaves * kJoinDeep) {
            float x[kJoinDeep];                      // (no condition on a load: it would be waited for before the next)
#pragma unroll
            for (int u = 0; u < kJoinDeep; ++u) x[u] = from[static_cast<int64_t>(min(k + u * kJoinWaves, a.chunks - 1)) * 2 * a.width];
#pragma unroll
            for (int u = 0; u < kJoinDeep; ++u) sum += k + u * kJoinWaves < a.chunks ? x[u] : 0.0f;
        }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= a.width) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) sum += part[w][lane];
    put_grad(out, a.grad, c, a.add, sum);
}

// ---- host ----

constexpr int kRowBlocks = 1 << 16;
// Parts and columns that the last block joins, in place of another launch: 8 x 256 5.7 us, 30 x 500 7.3, both 8.2 in two launches; one row of 4096, which
// is 16 columns a thread one after the other, 18.6.
constexpr int64_t kJoinParts = 4096, kJoinColumns = 512;

// Forward: a block for every row group (16384 x 1024 21.1 us, 1536 blocks that go on 22.4); teams of eight waves and more go on, which keeps
// their parameters in registers (4096 x 8192 48.7 us, a block a row 51.9).  Elements a lane: forward 16 (without residual 12.4 us, 8: 14.4), backward 8, which
// leaves room for the sums and another wave (20011 x 771 34.9 us, 16: 41.4).
constexpr int kForwardThreads = 256, kForwardBlocks = 1 << 20, kForwardWideBlocks = 1536, kBackwardThreads = 512, kForwardEach = 16, kBackwardEach = 8;

// The team of a width, as a type; false: rows are too short for a vector, or too long for a team.
template <int XT, int YT, int THREADS, int EACH, typename F>
bool with_team(int64_t width, F f) {
    constexpr int N = XT == DDP_FP32 ? 4 : 8;
    if (width < N || width > 16 * 64 * kMostEach) return false;
    if (width <= 4 * N) f(Team<XT, YT, 4, 1, THREADS, N>(0));
    else if (width <= 8 * N) f(Team<XT, YT, 8, 1, THREADS, N>(0));
    else if (width <= 8 * EACH) f(Team<XT, YT, 8, 1, THREADS, EACH>(0));
    else if (width <= 32 * EACH) f(Team<XT, YT, 32, 1, THREADS, EACH>(0));
    else if (width <= 64 * EACH) f(Team<XT, YT, 64, 1, THREADS, EACH>(0));
    else if (width <= 2 * 64 * EACH) f(Team<XT, YT, 64, 2, THREADS, EACH>(0));
    else if (width <= 4 * 64 * EACH) f(Team<XT, YT, 64, 4, THREADS, EACH>(0));
    else if (width <= 8 * 64 * EACH) f(Team<XT, YT, 64, 8, std::max(512, THREADS), EACH>(0));
    else if (width <= 16 * 64 * EACH) f(Team<XT, YT, 64, 16, 1024, EACH>(0));
    else f(Team<XT, YT, 64, 16, 1024, kMostEach>(0));
    return true;
}

template <int XT, int YT>
hipError_t launch_forward(ddp_layernorm* h, const ForwardArgs& a) {
    const bool team = with_team<XT, YT, kForwardThreads, kForwardEach>(a.width, [&](auto t) {
        typedef decltype(t) T;
        const int64_t blocks = std::min<int64_t>((a.rows + T::TEAMS - 1) / T::TEAMS, T::WAVES < 8 ? kForwardBlocks : kForwardWideBlocks);
        hipLaunchKernelGGL((forward_team_kernel<XT, YT, T>), dim3(static_cast<unsigned>(blocks)), dim3(T::THREADS), 0, h->stream, a);
    });
    if (!team)
        hipLaunchKernelGGL((forward_kernel<XT, YT>), dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kRowBlocks))), dim3(kThreads), 0, h->stream, a);
    return hipGetLastError();
}
// Returns the row chunks that sums are left of, -1 where they are joined already.
template <int XT, int YT>
int32_t launch_backward(ddp_layernorm* h, BackwardArgs a) {
    int32_t chunks = a.chunks;
    const bool team = with_team<XT, YT, kBackwardThreads, kBackwardEach>(a.width, [&](auto t) {
        typedef decltype(t) T;
        chunks = static_cast<int32_t>(std::min<int64_t>((a.rows + T::TEAMS - 1) / T::TEAMS, h->chunks));
        if (a.partial != nullptr && a.width <= kJoinColumns && static_cast<int64_t>(chunks) * 2 * a.width <= kJoinParts) a.counter = h->counter;
        hipLaunchKernelGGL((backward_team_kernel<XT, YT, T>), dim3(static_cast<unsigned>(chunks)), dim3(T::THREADS), 0, h->stream, a);
    });
    if (team) return a.counter != nullptr ? -1 : chunks;
    if (a.dx != nullptr)
        hipLaunchKernelGGL((backward_rows_kernel<XT, YT>), dim3(static_cast<unsigned>(std::min<int64_t>(a.rows, kRowBlocks))), dim3(kThreads), 0, h->stream, a);
    if (a.partial != nullptr)
        hipLaunchKernelGGL((backward_columns_kernel<XT, YT>), dim3(static_cast<unsigned>((a.width + 64 * kN - 1) / (64 * kN)), static_cast<unsigned>(a.chunks)),
                           dim3(kThreads), 0, h->stream, a);
    return chunks;
}

// y has x's type, or any where x is binary32.
bool known_pair(int xt, int yt) { return xt == DDP_FP32 || xt == yt; }
template <typename F>
auto with_types(int xt, int yt, F f) {
    if (xt == DDP_FP16) return f(std::integral_constant<int, DDP_FP16>(), std::integral_constant<int, DDP_FP16>());
    if (xt == DDP_BF16) return f(std::integral_constant<int, DDP_BF16>(), std::integral_constant<int, DDP_BF16>());
    if (yt == DDP_FP32) return f(std::integral_constant<int, DDP_FP32>(), std::integral_constant<int, DDP_FP32>());
    if (yt == DDP_FP16) return f(std::integral_constant<int, DDP_FP32>(), std::integral_constant<int, DDP_FP16>());
    return f(std::integral_constant<int, DDP_FP32>(), std::integral_constant<int, DDP_BF16>());
}

int32_t check_rows(ddp_layernorm* h, int64_t rows, int x_dtype, int y_dtype, int param_dtype) {
    if (rows < 0 || rows > kMaxRows) return layer_fail(h, DDP_ERR_ARG, "layer norm: rows outside [0, 2^31 - 1]");
    if (!known_dtype(x_dtype) || !known_dtype(y_dtype) || !known_dtype(param_dtype)) return layer_fail(h, DDP_ERR_ARG, "layer norm: unknown dtype");
    if (!known_pair(x_dtype, y_dtype)) return layer_fail(h, DDP_ERR_UNSUPPORTED, "layer norm: y of another 16-bit type than x, or binary32 for 16-bit x");
    return DDP_OK;
}
bool bad_stride(const ddp_layernorm* h, const void* p, int64_t stride) { return p && (stride < h->width || stride > INT32_MAX); }

}  // namespace

extern "C" {

const char* ddp_layernorm_last_error(const ddp_layernorm* h) { return h ? h->err.c_str() : ddp_last_error(nullptr); }

int32_t ddp_layernorm_create(ddp_layernorm** out, int32_t device, void* stream, int64_t width) {
    if (!out) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_layernorm_create: out is null");
    *out = nullptr;
    const int32_t status = layer_device("ddp_layernorm_create: bad device", device);
    if (status != DDP_OK) return status;
    if (width < 1) return layer_fail(nullptr, DDP_ERR_ARG, "ddp_layernorm_create: the width is at least 1");
    if (width > kMaxWidth) return layer_fail(nullptr, DDP_ERR_UNSUPPORTED, "ddp_layernorm_create: more than 2^20 columns");
    ddp_layernorm* h = new (std::nothrow) ddp_layernorm();
    if (!h) return layer_fail(nullptr, DDP_ERR_HIP, "out of host memory");
    h->device = device;
    h->stream = static_cast<hipStream_t>(stream);
    h->width = width;
    // two blocks a compute unit, one of the widest teams (32768 x 4096: 512 chunks 195 us, 256 213; 2048 x 12000: 256 53.6, 512 70.7)
    h->chunks = static_cast<int32_t>(std::max<int64_t>(16, std::min<int64_t>(width <= 8 * 1024 ? 512 : 256, (int64_t(1) << 22) / width)));
    if (device != DDP_DEVICE_NONE) {
        const int64_t sums = static_cast<int64_t>(h->chunks) * 2 * width * 4;
        hipError_t err = layer_alloc(h, sums + 256);
        if (err == hipSuccess) {
            OnDevice on(device);
            const uint32_t none = 0;
            err = taken(hipMemcpy(h->mem + sums, &none, sizeof none, hipMemcpyHostToDevice));
            if (err != hipSuccess) (void)taken(hipFree(h->mem));
        }
        if (err != hipSuccess) {
            delete h;
            return layer_fail(nullptr, DDP_ERR_HIP, hipGetErrorString(err));
        }
        h->partial = reinterpret_cast<float*>(h->mem);
        h->counter = reinterpret_cast<uint32_t*>(h->mem + sums);
    }
    *out = h;
    return DDP_OK;
}

int32_t ddp_layernorm_destroy(ddp_layernorm* h) {
    if (!h) return DDP_ERR_ARG;
    layer_release(h);
    delete h;
    return DDP_OK;
}

int32_t ddp_layernorm_forward(ddp_layernorm* h, int64_t rows, const void* x, int32_t x_dtype, int64_t x_stride, const void* residual,
                              int64_t residual_stride, const void* gamma, const void* beta, int32_t param_dtype, float eps, void* sum,
                              int64_t sum_stride, void* y, int32_t y_dtype, int64_t y_stride, float* mean, float* rstd) {
    if (!h) return DDP_ERR_ARG;
    const int32_t status = check_rows(h, rows, x_dtype, y_dtype, param_dtype);
    if (status != DDP_OK) return status;
    if (!(eps >= 0.0f)) return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_forward: eps below 0 or not a number");
    if (x_stride < h->width || x_stride > INT32_MAX || y_stride < h->width || y_stride > INT32_MAX || bad_stride(h, residual, residual_stride) ||
        bad_stride(h, sum, sum_stride))
        return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_forward: a stride is below the width (or above 2^31 - 1)");
    if (rows > 0 && (!x || !y)) return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_forward: null pointer");
    const int xs = elem_bytes(x_dtype), ps = elem_bytes(param_dtype);
    if (misaligned(x, xs) || misaligned(residual, xs) || misaligned(sum, xs) || misaligned(y, elem_bytes(y_dtype)) || misaligned(gamma, ps) ||
        misaligned(beta, ps) || misaligned(mean, 4) || misaligned(rstd, 4))
        return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_forward: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_layernorm_forward without a device");
    if (rows == 0) return DDP_OK;
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    ForwardArgs a{};
    a.x = static_cast<const char*>(x);
    a.residual = static_cast<const char*>(residual);
    a.gamma = static_cast<const char*>(gamma);
    a.beta = static_cast<const char*>(beta);
    a.sum = static_cast<char*>(sum);
    a.y = static_cast<char*>(y);
    a.mean = mean;
    a.rstd = rstd;
    a.rows = rows;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.sum_stride = sum_stride;
    a.y_stride = y_stride;
    a.width = static_cast<int32_t>(h->width);
    a.param = param_dtype;
    a.eps = eps;
    a.stream = rows * h->width * elem_bytes(y_dtype) >= kStreamBytes;
    LAYER_HIP(h, with_types(x_dtype, y_dtype, [&](auto xt, auto yt) { return launch_forward<xt.value, yt.value>(h, a); }));
    return DDP_OK;
}

int32_t ddp_layernorm_backward(ddp_layernorm* h, int64_t rows, const void* dy, int32_t dy_dtype, int64_t dy_stride, const void* x, int32_t x_dtype,
                               int64_t x_stride, const float* mean, const float* rstd, const void* gamma, int32_t param_dtype, const void* dsum,
                               int64_t dsum_stride, void* dx, int64_t dx_stride, int32_t accumulate, void* dgamma, void* dbeta, int32_t grad_dtype) {
    if (!h) return DDP_ERR_ARG;
    const int32_t status = check_rows(h, rows, x_dtype, dy_dtype, param_dtype);
    if (status != DDP_OK) return status;
    if (!known_dtype(grad_dtype)) return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_backward: unknown dtype");
    if (dy_stride < h->width || dy_stride > INT32_MAX || x_stride < h->width || x_stride > INT32_MAX || bad_stride(h, dsum, dsum_stride) ||
        bad_stride(h, dx, dx_stride))
        return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_backward: a stride is below the width (or above 2^31 - 1)");
    if (rows > 0 && (!dy || !x || !mean || !rstd)) return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_backward: null pointer");
    const int xs = elem_bytes(x_dtype), gs = elem_bytes(grad_dtype);
    if (misaligned(dy, elem_bytes(dy_dtype)) || misaligned(x, xs) || misaligned(dsum, xs) || misaligned(dx, xs) || misaligned(gamma, elem_bytes(param_dtype)) ||
        misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dgamma, gs) || misaligned(dbeta, gs))
        return layer_fail(h, DDP_ERR_ARG, "ddp_layernorm_backward: pointer not aligned to its element size");
    if (h->device == DDP_DEVICE_NONE) return layer_fail(h, DDP_ERR_NO_DEVICE, "ddp_layernorm_backward without a device");
    const bool params = dgamma || dbeta;
    if ((rows == 0 || !dx) && (!params || (rows == 0 && accumulate))) return DDP_OK;
    OnDevice on(h->device);
    LAYER_HIP(h, on.err);
    BackwardArgs a{};
    a.dy = static_cast<const char*>(dy);
    a.x = static_cast<const char*>(x);
    a.gamma = static_cast<const char*>(gamma);
    a.dsum = static_cast<const char*>(dsum);
    a.mean = mean;
    a.rstd = rstd;
    a.dx = static_cast<char*>(dx);
    a.partial = params ? h->partial : nullptr;
    a.dgamma = static_cast<char*>(dgamma);
    a.dbeta = static_cast<char*>(dbeta);
    a.grad = grad_dtype;
    a.add = accumulate != 0;
    a.rows = rows;
    a.dy_stride = dy_stride;
    a.x_stride = x_stride;
    a.dsum_stride = dsum_stride;
    a.dx_stride = dx_stride;
    a.rows_per_chunk = std::max<int64_t>(64, (rows + h->chunks - 1) / h->chunks);
    a.chunks = static_cast<int32_t>((rows + a.rows_per_chunk - 1) / a.rows_per_chunk);
    a.width = static_cast<int32_t>(h->width);
    a.param = param_dtype;
    a.stream = rows * h->width * elem_bytes(x_dtype) >= kStreamBytes;
    int32_t chunks = 0;
    if (rows > 0) {
        chunks = with_types(x_dtype, dy_dtype, [&](auto xt, auto yt) { return launch_backward<xt.value, yt.value>(h, a); });
        LAYER_HIP(h, hipGetLastError());
    }
    if (!params || chunks < 0) return DDP_OK;
    JoinArgs j{h->partial, static_cast<char*>(dgamma), static_cast<char*>(dbeta), a.width, chunks, grad_dtype, accumulate != 0};
    hipLaunchKernelGGL(join_kernel, dim3(static_cast<unsigned>((a.width + 63) / 64), 2), dim3(64 * kJoinWaves), 0, h->stream, j);
    LAYER_HIP(h, hipGetLastError());
    return DDP_OK;
}

}  // extern "C"
