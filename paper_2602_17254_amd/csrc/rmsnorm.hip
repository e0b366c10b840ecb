// Root-mean-square norm over the rows of [ranks][tokens][width], after a residual's addition, and its gradients.
//
//   s = x + residual      rstd = 1 / sqrt(sum s^2 / width + eps)      y = s rstd gamma
//   in 8 bits: scale = max |y| / 448 per row, y / scale rounded to e4m3
//
//   h = s rstd      g = gamma dy      dx = rstd (g - h sum(g h) / width) + dtotal
//   dgamma = sum over a rank's tokens of dy h
//
// Memory bounds both directions. A row is held in registers by a group of lanes, so it is read once; a row has one
// sum (and one maximum with it: that of |s gamma|, as rstd is the same for the whole row), so one barrier where
// several waves hold it. A lane holds the same columns of every row: the weight gradients of a workgroup's rows add
// up in registers, go to the workspace, and are joined in a fixed order in 64 bits, as those of the layer norm.
// A lane adds up at most 32 values of a row in fp32, then lanes and waves their sums in some 22 steps: a sum is off by at most
// 54 roundings of the sum of its terms' sizes. The lanes of longer rows have many vectors, whose sums meet in 64 bits. y comes from the
// sum before it is rounded to the stored type; total, y and dx are rounded once.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "norm.h"
#include "operators.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

constexpr int64_t kBlocks = 32;  // of kThreads lanes, of the forward pass for each of the 256 CUs
constexpr float kLargest8 = 448.0f;                        // of e4m3
constexpr float kSmallestScale = 1.1754943508222875e-38f;  // 2^-126, so that one over it is a number

template <typename T>
struct Forward {
    const T *x, *residual;
    T* total;
    void* y;  // of T, or e4m3 with scales
    const void* gamma;
    float *rstd, *scales;
    int64_t ranks, tokens, width, x_rank, x_token, residual_rank, residual_token, total_rank, total_token, y_rank, y_token;
    float eps;
    int weight_type;
    bool stream;  // the tensors are larger than the caches
};

// A row's sum and maximum with one barrier; `slots` alternate from each row of a workgroup to its next, whatever
// their ranks. Where OUT8 is not set there is no maximum.
template <int LANES, bool MAX>
__device__ __forceinline__ void row_sum_max(float& sum, float& most, float2* slots) {
    sum = lanes_sum<LANES <= 64 ? LANES : 64>(sum);
    if constexpr (MAX) most = lanes_max<LANES <= 64 ? LANES : 64>(most);
    if constexpr (LANES > 64) {
        if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = make_float2(sum, most);
        __syncthreads();
        sum = most = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) {
            const float2 s = slots[w];
            sum += s.x;
            if constexpr (MAX) most = fmaxf(most, s.y);
        }
    }
}

// A value in 8 bits: beyond the largest number only by its factor's rounding, which the conversion would make NaN of.
__device__ __forceinline__ float within_8(float v) {
    return v > kLargest8 ? kLargest8 : v < -kLargest8 ? -kLargest8 : v;  // NaN stays
}

template <int V>
__device__ __forceinline__ auto to_8(const float (&v)[V]) {
    typedef uint8_t Bytes __attribute__((ext_vector_type(V), aligned(1)));
    if constexpr (V == 1) {
        return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(within_8(v[0]), 0.0f, 0, false);
    } else {
        typedef int Words __attribute__((ext_vector_type(V / 4)));
        Words w;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const int low = __builtin_amdgcn_cvt_pk_fp8_f32(within_8(v[4 * i]), within_8(v[4 * i + 1]), 0, false);
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(within_8(v[4 * i + 2]), within_8(v[4 * i + 3]), low, true);
        }
        return __builtin_bit_cast(Bytes, w);
    }
}

// The scale of a row whose largest value is `most` before rstd, and one over it. A row that holds a NaN has a NaN
// for both.
__device__ __forceinline__ float2 scale_of(float most, float rstd) {
    const float scale = __builtin_elementwise_maximum(most * rstd / kLargest8, kSmallestScale);
    return make_float2(scale, 1.0f / scale);
}

// Bound by the bytes of its rows: 8 x 4096 x 4096 bf16 with a residual 179 us (1074 MB, 6.0 TB/s, where a copy reaches 6.8), to 8 bits 156
// (940 MB, 6.0). A row's next load is on its way during its sum. One token of 4096 takes 2.9 us, the latency of one load and one
// sum. STREAM: the tensors would not stay in the caches and go past them.
template <typename T, int V, int LANES, int NV, bool STREAM, bool OUT8>
__global__ __launch_bounds__(kBlock<LANES>) void rms_forward_kernel(Forward<T> a) {
    constexpr int G = kBlock<LANES> / LANES;
    __shared__ float2 slots[2][kWide / 64];
    const int lane = threadIdx.x % LANES, group = group_of_lane<LANES>();
    const Columns<V, LANES, NV> own(lane, (int)a.width);
    const float inv = 1.0f / (float)a.width;
    float gamma[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) load_weights<V>(a.gamma, a.weight_type, own.first[j], a.width, 1.0f, gamma[j]);
    struct Ahead {
        Some<T, V> x[NV], residual[NV];
    };
    const auto fetch = [&](int64_t r, int64_t t, Ahead& to) {
        const T* x = a.x + r * a.x_rank + t * a.x_token;
        const T* residual = a.residual + r * a.residual_rank + t * a.residual_token;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (own.skip[j] < V) {
                to.x[j] = load_vector<STREAM, V>(x + own.first[j]);
                if (a.residual) to.residual[j] = load_vector<STREAM, V>(residual + own.first[j]);
            }
    };
    const int64_t step = (int64_t)gridDim.x * G;
    int turn = 0;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        Ahead next;
        int64_t t = (int64_t)blockIdx.x * G + group;
        if (t < a.tokens) fetch(r, t, next);
        for (; t < a.tokens; t += step) {  // whole groups of lanes, whole workgroups where a row takes one
            float v[NV][V], most = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    v[j][k] = (float)next.x[j][k];
                    if (a.residual) v[j][k] += (float)next.residual[j][k];
                }
            if (t + step < a.tokens) fetch(r, t + step, next);  // on its way during this row's sum
            float square = own.sum([&](int j, int k) { return v[j][k] * v[j][k]; });
            if constexpr (OUT8) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if (own.skip[j] < V) most = fmaxf(most, fabsf(v[j][k] * gamma[j][k]));
            }
            row_sum_max<LANES, OUT8>(square, most, slots[turn]);
            turn ^= 1;
            const float rstd = 1.0f / sqrtf(square * inv + a.eps);
            if (a.total) {
                T* total = a.total + r * a.total_rank + t * a.total_token;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Some<T, V> o;
#pragma unroll
                    for (int k = 0; k < V; ++k) o[k] = (T)v[j][k];
                    if (own.skip[j] < V) store_vector<STREAM, V>(total + own.first[j], o);
                }
            }
            const int64_t at = r * a.y_rank + t * a.y_token;
            if constexpr (OUT8) {
                const float2 by = scale_of(most, rstd);
                uint8_t* y = static_cast<uint8_t*>(a.y) + at;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float o[V];
#pragma unroll
                    for (int k = 0; k < V; ++k) o[k] = v[j][k] * rstd * gamma[j][k] * by.y;
                    if (own.skip[j] < V) store_vector<STREAM, V>(y + own.first[j], to_8<V>(o));
                }
                if (lane == 0) a.scales[r * a.tokens + t] = by.x;
            } else {
                T* y = static_cast<T*>(a.y) + at;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Some<T, V> o;
#pragma unroll
                    for (int k = 0; k < V; ++k) o[k] = (T)(v[j][k] * rstd * gamma[j][k]);
                    if (own.skip[j] < V) store_vector<STREAM, V>(y + own.first[j], o);
                }
            }
            if (lane == 0 && a.rstd) a.rstd[r * a.tokens + t] = rstd;
        }
    }
}

// Rows beyond what a workgroup's registers hold: read twice, the second time from the caches. A lane adds up to 4096 vectors: one
// after another in fp32, rstd was off by 5e-5 of itself at 2^24 equal values. 8 x 1024 x 20001 bf16 223 us, of which the bytes take 96.
template <typename T, bool OUT8>
__global__ __launch_bounds__(kWide) void rms_forward_long_kernel(Forward<T> a) {
    constexpr int V = kVec<T>;
    __shared__ float2 slots[2][kWide / 64];
    const float inv = 1.0f / (float)a.width;
    const int64_t i0 = (int64_t)threadIdx.x * V;
    int turn = 0;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
            const T* x = a.x + r * a.x_rank + t * a.x_token;
            const T* residual = a.residual + r * a.residual_rank + t * a.residual_token;
            const auto fetch = [&](int64_t i, float(&v)[V]) {
                load_row<T>(x, i, a.width, 0.0f, v);
                if (a.residual) {
                    float w[V];
                    load_row<T>(residual, i, a.width, 0.0f, w);
#pragma unroll
                    for (int k = 0; k < V; ++k) v[k] += w[k];
                }
            };
            float v[V], gamma[V], most = 0.0f;
            double squares = 0.0;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                fetch(i, v);
                float part = 0.0f;
#pragma unroll
                for (int k = 0; k < V; ++k) part += v[k] * v[k];
                squares += part;
                if constexpr (OUT8) {
                    load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
#pragma unroll
                    for (int k = 0; k < V; ++k) most = fmaxf(most, fabsf(v[k] * gamma[k]));
                }
            }
            float square = (float)squares;
            row_sum_max<kWide, OUT8>(square, most, slots[turn]);
            turn ^= 1;
            const float rstd = 1.0f / sqrtf(square * inv + a.eps);
            const float2 by = OUT8 ? scale_of(most, rstd) : make_float2(0.0f, 0.0f);
            const int64_t at = r * a.y_rank + t * a.y_token;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                fetch(i, v);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
                if (a.total) store_row<T, V>(a.total + r * a.total_rank + t * a.total_token, i, a.width, v);
                if constexpr (OUT8) {
                    uint8_t* y = static_cast<uint8_t*>(a.y) + at;
#pragma unroll
                    for (int k = 0; k < V; ++k) v[k] = v[k] * rstd * gamma[k] * by.y;
                    const auto o = to_8<V>(v);
                    if (i + V <= a.width) {
                        store_vector<false, V>(y + i, o);
                    } else {
#pragma unroll
                        for (int k = 0; k < V; ++k)
                            if (i + k < a.width) y[i + k] = o[k];
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < V; ++k) v[k] = v[k] * rstd * gamma[k];
                    store_row<T, V>(static_cast<T*>(a.y) + at, i, a.width, v);
                }
            }
            if (threadIdx.x == 0) {
                if (a.rstd) a.rstd[r * a.tokens + t] = rstd;
                if (OUT8) a.scales[r * a.tokens + t] = by.x;
            }
        }
    }
}

template <typename T>
struct Backward {
    const T *dy, *total, *dtotal;
    T* dx;
    const void* gamma;
    const float* rstd;
    float* dgamma;  // rows `grad_rank` apart
    float* parts;   // [ranks][chunks][width], where a rank's tokens are in several chunks
    int64_t ranks, tokens, width, dy_rank, dy_token, total_rank, total_token, dtotal_rank, dtotal_token, dx_rank, dx_token,
        grad_rank;
    int64_t chunks;  // of a rank's tokens: every chunk takes every chunks-th group of rows
    int weight_type;
    bool stream;  // the tensors are larger than the caches
};

// Where a chunk's sums go, if anywhere: the rank's own gradient where it is the only one.
template <typename T>
__device__ __forceinline__ float* sums_of(const Backward<T>& a, int64_t r, int64_t c) {
    if (!a.dgamma) return nullptr;
    return a.chunks > 1 ? a.parts + (r * a.chunks + c) * a.width : a.dgamma + r * a.grad_rank;
}

// Bound by the bytes of its rows: 376 us at 8 x 4096 x 8192 bf16 with dtotal, 2.15 GB, 5.7 TB/s (and 7 us to join the workgroups' sums). The rows
// of a rank go to its workgroups in turn, so that those at work read neighbouring rows: with consecutive rows of its own for each it
// took 390, and 5 to 13% more on 8 of 10 sizes (2 to 9% less on 8 x 4096 x 2048 and 8 x 16384 x 512). Loads a row ahead make no difference there,
// but 5% at 9 x 777 x 1283 fp16, 16 us and 4 to join. Rows of 8193 to 16384 values leave no registers for all of it: 20 to 100 bytes of
// a lane go to scratch memory. 8 x 4096 x 16384 bf16 takes 770 us, 5.6 TB/s, 8 x 1024 x 16384 fp32 385, 5.6, but 8 x 1024 x 8200 bf16,
// whose lanes' third and fourth vectors are void but for one, 112, 4.8.
template <typename T, int V, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(kBlock<LANES>, (kLocalGamma<V, LANES, NV> ? 4 : 1)) void rms_backward_kernel(Backward<T> a) {
    constexpr int G = kBlock<LANES> / LANES;
    __shared__ float slots[2][kWide / 64];
    __shared__ float join[G > 1 ? kThreads * NV * V : 1];
    const int lane = threadIdx.x % LANES, group = group_of_lane<LANES>();
    const Columns<V, LANES, NV> own(lane, (int)a.width);
    const float inv = 1.0f / (float)a.width;
    constexpr bool kLocal = kLocalGamma<V, LANES, NV>;
    __shared__ float gammas[kLocal ? LANES * NV * V : 1];
    float gamma[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) load_weights<V>(a.gamma, a.weight_type, own.first[j], a.width, 1.0f, gamma[j]);
    if constexpr (kLocal) {  // each lane reads only what it wrote
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) gammas[(j * LANES + lane) * V + k] = gamma[j][k];
    }
    int turn = 0;  // goes on from one rank to the next: no barrier stands between their rows
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t c = blockIdx.x;
        float dg[NV][V] = {};
        struct Ahead {
            Some<T, V> total[NV], dy[NV], dtotal[NV];
            float rstd;
        };
        const auto fetch = [&](int64_t t, Ahead& to) {
            const T* total = a.total + r * a.total_rank + t * a.total_token;
            const T* dy = a.dy + r * a.dy_rank + t * a.dy_token;
            const T* dtotal = a.dtotal + r * a.dtotal_rank + t * a.dtotal_token;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (own.skip[j] < V) {
                    to.total[j] = load_vector<STREAM, V>(total + own.first[j]);
                    to.dy[j] = load_vector<STREAM, V>(dy + own.first[j]);
                    if (a.dtotal) to.dtotal[j] = load_vector<STREAM, V>(dtotal + own.first[j]);
                }
            to.rstd = a.rstd[r * a.tokens + t];
        };
        const int64_t step = a.chunks * G;
        // the next row is on its way during this row's sum, where there are registers for both
        constexpr bool kAhead = NV * V * sizeof(T) <= 64;
        const auto row = [&](int64_t t, Ahead& next) {
            if (!kAhead) fetch(t, next);
            float rstd = next.rstd;
            if constexpr (LANES >= 64)  // the same in a wave: in a scalar register
                rstd = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, rstd)));
            float h[NV][V], g[NV][V];
            Some<T, V> more[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                more[j] = next.dtotal[j];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    h[j][k] = (float)next.total[j][k] * rstd;
                    g[j][k] = (float)next.dy[j][k];
                    dg[j][k] += g[j][k] * h[j][k];
                    g[j][k] *= kLocal ? gammas[(j * LANES + lane) * V + k] : gamma[j][k];
                }
            }
            if (kAhead && t + step < a.tokens) fetch(t + step, next);
            const float along = inv * row_sum<LANES>(own.sum([&](int j, int k) { return g[j][k] * h[j][k]; }), slots[turn]);
            turn ^= 1;
            T* dx = a.dx + r * a.dx_rank + t * a.dx_token;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Some<T, V> o;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    float d = rstd * (g[j][k] - h[j][k] * along);
                    if (a.dtotal) d += (float)more[j][k];
                    o[k] = (T)d;
                }
                if (own.skip[j] < V) store_vector<STREAM, V>(dx + own.first[j], o);
            }
        };
        Ahead next;
        int64_t t = c * G + group;
        if (kAhead && t < a.tokens) fetch(t, next);
        for (; t < a.tokens; t += step) row(t, next);
        float* out = sums_of(a, r, c);
        if (!out) continue;
        if constexpr (G == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Some<float, V> o;
#pragma unroll
                for (int k = 0; k < V; ++k) o[k] = dg[j][k];
                if (own.skip[j] < V) *reinterpret_cast<Some<float, V>*>(out + own.first[j]) = o;
            }
        } else {
            // the groups' sums, in the groups' order
            constexpr int N = LANES * NV * V;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (own.skip[j] < V) join[group * N + own.first[j] + k] = dg[j][k];
            __syncthreads();
            for (int i = threadIdx.x; i < N && i < a.width; i += kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < G; ++q) s += join[q * N + i];
                out[i] = s;
            }
        }
    }
}

// Rows beyond what a workgroup's registers hold: read twice, the second time from the caches, the sum of their vectors' sums
// in 64 bits, and the chunk's sums of the weight gradients added up where they go. 8 x 1024 x 20001 bf16 863 us, 651 without
// dgamma, where the bytes take 145: a lane's loads wait for those before.
template <typename T>
__global__ __launch_bounds__(kWide) void rms_backward_long_kernel(Backward<T> a) {
    constexpr int V = kVec<T>;
    __shared__ double slots[2][kWide / 64];
    const float inv = 1.0f / (float)a.width;
    const int64_t i0 = (int64_t)threadIdx.x * V;
    int turn = 0;  // goes on from one rank to the next
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t c = blockIdx.x;
        float* dgamma = sums_of(a, r, c);
        // a lane adds to the same columns for every row
        for (int64_t i = i0; dgamma && i < a.width; i += kWide * V) {
            const float zero[V] = {};
            store_row<float, V>(dgamma, i, a.width, zero);
        }
        for (int64_t t = c; t < a.tokens; t += a.chunks) {
            const T* total = a.total + r * a.total_rank + t * a.total_token;
            const T* dy = a.dy + r * a.dy_rank + t * a.dy_token;
            const T* dtotal = a.dtotal + r * a.dtotal_rank + t * a.dtotal_token;
            T* dx = a.dx + r * a.dx_rank + t * a.dx_token;
            const float rstd = a.rstd[r * a.tokens + t];
            float h[V], g[V], gamma[V];
            double sum = 0.0;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                load_row<T>(total, i, a.width, 0.0f, h);
                load_row<T>(dy, i, a.width, 0.0f, g);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
                float part = 0.0f;
#pragma unroll
                for (int k = 0; k < V; ++k) part += g[k] * gamma[k] * (h[k] * rstd);
                sum += part;
            }
            const float along = inv * (float)row_sum<kWide>(sum, slots[turn]);
            turn ^= 1;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                float o[V], more[V] = {};
                load_row<T>(total, i, a.width, 0.0f, h);
                load_row<T>(dy, i, a.width, 0.0f, g);
                if (a.dtotal) load_row<T>(dtotal, i, a.width, 0.0f, more);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    h[k] *= rstd;
                    o[k] = rstd * (g[k] * gamma[k] - h[k] * along) + more[k];
                }
                store_row<T, V>(dx, i, a.width, o);
                if (dgamma) {
                    float s[V];
                    load_values<float, V>(dgamma, i, a.width, 0.0f, s);
#pragma unroll
                    for (int k = 0; k < V; ++k) s[k] += g[k] * h[k];
                    store_row<float, V>(dgamma, i, a.width, s);
                }
            }
        }
    }
}

// Besides the layer norm's shapes, for 16-bit rows of 129 to 256 vectors, 256 lanes with one vector each: a second one would be void
// for most of them. 9 x 777 x 1283 fp16 forward 16.5 us in place of 20.5, 8 x 8192 x 1100 bf16 to 8 bits 140 in place of 175, backward 94 in
// place of 119.
template <typename T>
bool one_vector(int64_t width) {
    const int64_t n = (width + kVec<T> - 1) / kVec<T>;
    return kVec<T> == 8 && n > 128 && n <= 256;
}

// Workgroups of the forward pass: a few times what the GPU holds, with the same number of rows each, so that
// the weights are loaded once for all of them and a row's load overlaps the one before.
template <typename T, bool OUT8>
int run_forward(Forward<T> a, hipStream_t stream) {
    const auto dense = [&](const void* p, int64_t rank, int64_t token) { return !p || rank == a.tokens * token; };
    if (dense(a.x, a.x_rank, a.x_token) && dense(a.residual, a.residual_rank, a.residual_token) &&
        dense(a.total, a.total_rank, a.total_token) && dense(a.y, a.y_rank, a.y_token)) {  // rank after rank
        a.tokens *= a.ranks;
        a.ranks = 1;
    }
    const Shape shape = shape_of<T>(a.width);
    const int64_t units = (a.tokens + group_rows(shape) - 1) / group_rows(shape);
    const int64_t most = imax(1, 256 * kBlocks * kThreads / block_lanes(shape) / a.ranks);
    int64_t each = (units + most - 1) / most;
    // of many rows shorter workgroups: 8 x 4096 x 4096 bf16 179 us in place of 185, 2 to 6% on 12 of 14 sizes
    if (each >= 4) each = (each + 1) / 2;
    const dim3 grid((unsigned)((units + each - 1) / each), (unsigned)imin(a.ranks, kMaxGridY));
#define RUN(V, L, N)                                                                           \
    if (a.stream) rms_forward_kernel<T, V, L, N, true, OUT8><<<grid, kBlock<L>, 0, stream>>>(a); \
    else rms_forward_kernel<T, V, L, N, false, OUT8><<<grid, kBlock<L>, 0, stream>>>(a)
#define RUN_LONG() rms_forward_long_kernel<T, OUT8><<<grid, kWide, 0, stream>>>(a)
    if (one_vector<T>(a.width)) {
        RUN(kVec<T>, 256, 1);
        return launch_status();
    }
    TRIVANCE_NORM_SHAPES(RUN, RUN_LONG)
#undef RUN
#undef RUN_LONG
    return launch_status();
}

template <typename T>
int run_backward(const Backward<T>& a, hipStream_t stream) {
    const Shape shape = shape_of<T>(a.width);
    const dim3 grid((unsigned)a.chunks, (unsigned)imin(a.ranks, kMaxGridY));
#define RUN(V, L, N)                                                                      \
    if (a.stream) rms_backward_kernel<T, V, L, N, true><<<grid, kBlock<L>, 0, stream>>>(a); \
    else rms_backward_kernel<T, V, L, N, false><<<grid, kBlock<L>, 0, stream>>>(a)
#define RUN_LONG() rms_backward_long_kernel<T><<<grid, kWide, 0, stream>>>(a)
    if (one_vector<T>(a.width)) {
        RUN(kVec<T>, 256, 1);
    } else {
        TRIVANCE_NORM_SHAPES(RUN, RUN_LONG)
    }
#undef RUN
#undef RUN_LONG
    const int rc = launch_status();
    if (rc || a.chunks == 1 || !a.dgamma) return rc;
    return join_chunks(a.parts, a.dgamma, nullptr, 1, a.ranks, a.chunks, a.width, a.grad_rank, stream);
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" {

int trivance_rmsnorm_forward(const void* x, const void* residual, const void* gamma, void* total, void* y,
                             float* rstd, float* scales, int64_t ranks, int64_t tokens, int64_t width,
                             int64_t x_rank_stride, int64_t x_token_stride, int64_t residual_rank_stride,
                             int64_t residual_token_stride, int64_t total_rank_stride, int64_t total_token_stride,
                             int64_t y_rank_stride, int64_t y_token_stride, double eps, int dtype, int y_dtype,
                             int weight_dtype, void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype)) return TRIVANCE_EINVAL;
    if (y_dtype != dtype && y_dtype != TRIVANCE_E4M3) return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, width) || !(eps >= 0.0)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    const auto fits = [&](int64_t rank, int64_t token) { return rows_fit(ranks, tokens, width, rank, token); };
    const auto written = [&](int64_t rank, int64_t token) {
        return fits(rank, token) && rows_distinct(ranks, tokens, width, rank, token);
    };
    if (!x || !y || y == total || !fits(x_rank_stride, x_token_stride) || !written(y_rank_stride, y_token_stride) ||
        (residual && !fits(residual_rank_stride, residual_token_stride)) ||
        (total && !written(total_rank_stride, total_token_stride)))
        return TRIVANCE_EINVAL;
    const auto in_place = [&](const void* out, int64_t rank, int64_t token) {
        return rows_in_place(out, x, ranks, tokens, rank, token, x_rank_stride, x_token_stride) &&
               (!residual ||
                rows_in_place(out, residual, ranks, tokens, rank, token, residual_rank_stride, residual_token_stride));
    };
    if (!in_place(y, y_rank_stride, y_token_stride) || !in_place(total, total_rank_stride, total_token_stride))
        return TRIVANCE_EINVAL;
    const bool out8 = y_dtype == TRIVANCE_E4M3;
    // scales go with 8 bits, whose rows cannot take the place of wider ones
    if (out8 ? !scales || y == x || y == residual : scales != nullptr) return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        const Forward<T> a{static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(total), y, gamma,
                           rstd, scales, ranks, tokens, width, x_rank_stride, x_token_stride, residual_rank_stride,
                           residual_token_stride, total_rank_stride, total_token_stride, y_rank_stride, y_token_stride,
                           (float)eps, weight_dtype, ranks * tokens * width * (int64_t)sizeof(T) > kStreamBytes};
        return out8 ? run_forward<T, true>(a, s) : run_forward<T, false>(a, s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

int64_t trivance_rmsnorm_workspace_bytes(int64_t ranks, int64_t tokens, int64_t width) {
    if (!sizes_ok(ranks, tokens, width)) return TRIVANCE_EINVAL;
    int64_t most = 0;
    for (const int dtype : {TRIVANCE_F32, TRIVANCE_BF16}) {
        const int64_t per = chunk_tokens(ranks, tokens, shape_of(width, dtype));
        const int64_t chunks = imax(1, (tokens + per - 1) / per);
        if (chunks > 1) most = imax(most, ranks * chunks * width * (int64_t)sizeof(float));
    }
    return most;
}

int trivance_rmsnorm_backward(const void* dy, const void* total, const void* gamma, const float* rstd,
                              const void* dtotal, void* dx, float* dgamma, int64_t ranks, int64_t tokens,
                              int64_t width, int64_t dy_rank_stride, int64_t dy_token_stride,
                              int64_t total_rank_stride, int64_t total_token_stride, int64_t dtotal_rank_stride,
                              int64_t dtotal_token_stride, int64_t dx_rank_stride, int64_t dx_token_stride,
                              int64_t grad_rank_stride, int dtype, int weight_dtype, void* workspace,
                              int64_t workspace_bytes, void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype)) return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, width)) return TRIVANCE_EINVAL;
    if (dgamma && !(rows_fit(ranks, 1, width, grad_rank_stride, 0) && rows_distinct(ranks, 1, width, grad_rank_stride, 0)))
        return TRIVANCE_EINVAL;
    const auto fits = [&](int64_t rank, int64_t token) { return rows_fit(ranks, tokens, width, rank, token); };
    if (tokens > 0 && (!dy || !total || !rstd || !dx || !fits(dy_rank_stride, dy_token_stride) ||
                       !fits(total_rank_stride, total_token_stride) || !fits(dx_rank_stride, dx_token_stride) ||
                       (dtotal && !fits(dtotal_rank_stride, dtotal_token_stride)) ||
                       !rows_distinct(ranks, tokens, width, dx_rank_stride, dx_token_stride)))
        return TRIVANCE_EINVAL;
    const auto in_place = [&](const void* in, int64_t rank, int64_t token) {
        return rows_in_place(dx, in, ranks, tokens, dx_rank_stride, dx_token_stride, rank, token);
    };
    if (tokens > 0 && !(in_place(dy, dy_rank_stride, dy_token_stride) && in_place(total, total_rank_stride, total_token_stride) &&
                        (!dtotal || in_place(dtotal, dtotal_rank_stride, dtotal_token_stride))))
        return TRIVANCE_EINVAL;
    const int64_t need = trivance_rmsnorm_workspace_bytes(ranks, tokens, width);
    if (dgamma && (workspace_bytes < need || (need > 0 && !workspace))) return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(float)) return TRIVANCE_EINVAL;
    if (tokens == 0 && !dgamma) return TRIVANCE_OK;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        const int64_t per = chunk_tokens(ranks, tokens, shape_of<T>(width));
        return run_backward(
            Backward<T>{static_cast<const T*>(dy), static_cast<const T*>(total), static_cast<const T*>(dtotal),
                        static_cast<T*>(dx), gamma, rstd, dgamma, static_cast<float*>(workspace), ranks, tokens, width,
                        dy_rank_stride, dy_token_stride, total_rank_stride, total_token_stride, dtotal_rank_stride,
                        dtotal_token_stride, dx_rank_stride, dx_token_stride, grad_rank_stride,
                        imax(1, (tokens + per - 1) / per), weight_dtype,
                        ranks * tokens * width * (int64_t)sizeof(T) > kStreamBytes},
            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

}  // extern "C"
