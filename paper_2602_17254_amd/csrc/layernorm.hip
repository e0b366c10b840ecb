// Layer norm over the rows of [ranks][tokens][width], and its gradients.
//
//   mean = sum x / width      var = sum (x - mean)^2 / width      rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd       y = gamma h + beta
//
//   g = gamma dy      dx = rstd (g - sum g / width - h sum(g h) / width)
//   dgamma = sum over a rank's tokens of dy h      dbeta = sum over a rank's tokens of dy
//
// Memory bounds both directions. A row is held in registers by a group of lanes, so it is read once:
// the forward pass takes the mean and then the squares about it, the backward pass both row sums, from
// there. A lane holds the same columns of every row, so the weight gradients of a workgroup's
// rows add up in registers too; a workgroup's sums go to the workspace and a second kernel joins them
// in a fixed order, in 64 bits, into the rank's row. All sums are in fp32 or more, that of the mean in 64
// bits, as a row's values may nearly cancel; y and dx are rounded once.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "norm.h"
#include "operators.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

constexpr int64_t kBlocks = 32;  // of kThreads lanes, of the forward pass for each of the 256 CUs

template <typename T>
struct Forward {
    const T* x;
    T* y;
    const void *gamma, *beta;
    float *mean, *rstd;
    int64_t ranks, tokens, width, x_rank, x_token, y_rank, y_token;
    float eps;
    int weight_type;
    bool stream;  // the tensors are larger than the caches
};

// Bound by the bytes of x and y: 92 us at 8 x 4096 x 4096 bf16, 537 MB, 5.8 TB/s, where a copy of that size
// reaches 6.8. A row's next load is on its way during its sums; two rows ahead were slower, as were
// workgroups of 1024 lanes. STREAM: the tensors would not stay in the caches and go past them. One token of
// 4096 takes 3.4 us, the latency of one load and two sums.
template <typename T, int V, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(kBlock<LANES>) void norm_forward_kernel(Forward<T> a) {
    constexpr int G = kBlock<LANES> / LANES;
    __shared__ double sums[kWide / 64];
    __shared__ float squares[kWide / 64];
    const int lane = threadIdx.x % LANES, group = group_of_lane<LANES>();
    const Columns<V, LANES, NV> own(lane, (int)a.width);
    const float inv = 1.0f / (float)a.width;
    float gamma[NV][V], beta[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        load_weights<V>(a.gamma, a.weight_type, own.first[j], a.width, 1.0f, gamma[j]);
        load_weights<V>(a.beta, a.weight_type, own.first[j], a.width, 0.0f, beta[j]);
    }
    const auto fetch = [&](int64_t r, int64_t t, Some<T, V>(&to)[NV]) {
        const T* x = a.x + r * a.x_rank + t * a.x_token;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (own.skip[j] < V)
                to[j] = load_vector<STREAM, V>(x + own.first[j]);
    };
    const int64_t step = (int64_t)gridDim.x * G;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        Some<T, V> next[NV];
        int64_t t = (int64_t)blockIdx.x * G + group;
        if (t < a.tokens) fetch(r, t, next);
        for (; t < a.tokens; t += step) {  // whole groups of lanes, whole workgroups where a row takes one
            float v[NV][V];
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) v[j][k] = (float)next[j][k];
            if (t + step < a.tokens) fetch(r, t + step, next);  // on its way during this row's sums
            const float mean =
                (float)(row_sum<LANES>(own.sum([&](int j, int k) { return (double)v[j][k]; }), sums) / (double)a.width);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) v[j][k] -= mean;
            const float square =
                row_sum<LANES>(own.sum([&](int j, int k) { return v[j][k] * v[j][k]; }), squares);
            const float rstd = 1.0f / sqrtf(square * inv + a.eps);
            T* y = a.y + r * a.y_rank + t * a.y_token;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Some<T, V> o;
#pragma unroll
                for (int k = 0; k < V; ++k) o[k] = (T)(v[j][k] * rstd * gamma[j][k] + beta[j][k]);
                if (own.skip[j] < V) store_vector<STREAM, V>(y + own.first[j], o);
            }
            if (lane == 0) {
                if (a.mean) a.mean[r * a.tokens + t] = mean;
                if (a.rstd) a.rstd[r * a.tokens + t] = rstd;
            }
        }
    }
}

// Rows beyond what a workgroup's registers hold: read three times, the last two from the caches.
template <typename T>
__global__ __launch_bounds__(kWide) void norm_forward_long_kernel(Forward<T> a) {
    constexpr int V = kVec<T>;
    __shared__ double sums[kWide / 64];
    __shared__ float squares[kWide / 64];
    const float inv = 1.0f / (float)a.width;
    const int64_t i0 = (int64_t)threadIdx.x * V;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
            const T* x = a.x + r * a.x_rank + t * a.x_token;
            T* y = a.y + r * a.y_rank + t * a.y_token;
            float v[V], q = 0.0f;
            double s = 0.0;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                load_row<T>(x, i, a.width, 0.0f, v);
#pragma unroll
                for (int k = 0; k < V; ++k) s += v[k];
            }
            const float mean = (float)(row_sum<kWide>(s, sums) / (double)a.width);
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                load_row<T>(x, i, a.width, mean, v);
#pragma unroll
                for (int k = 0; k < V; ++k) q += (v[k] - mean) * (v[k] - mean);
            }
            const float rstd = 1.0f / sqrtf(row_sum<kWide>(q, squares) * inv + a.eps);
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                float gamma[V], beta[V];
                load_row<T>(x, i, a.width, 0.0f, v);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
                load_weights<V>(a.beta, a.weight_type, i, a.width, 0.0f, beta);
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] = (v[k] - mean) * rstd * gamma[k] + beta[k];
                store_row<T, V>(y, i, a.width, v);
            }
            if (threadIdx.x == 0) {
                if (a.mean) a.mean[r * a.tokens + t] = mean;
                if (a.rstd) a.rstd[r * a.tokens + t] = rstd;
            }
        }
    }
}

template <typename T>
struct Backward {
    const T *dy, *x;
    T* dx;
    const void* gamma;
    const float *mean, *rstd;
    float *dgamma, *dbeta;  // rows `grad_rank` apart
    float* parts;           // [ranks][chunks][2][width], where a rank's tokens are in several chunks
    int64_t ranks, tokens, width, dy_rank, dy_token, x_rank, x_token, dx_rank, dx_token, grad_rank;
    int64_t chunks, per;    // chunks of a rank's tokens, and the tokens of one
    int weight_type;
    bool stream;  // the tensors are larger than the caches
};

// Where a chunk's sums go, if anywhere: the rank's own gradients where it is the only one.
template <typename T>
__device__ __forceinline__ float* sums_of(const Backward<T>& a, int64_t r, int64_t c, int which) {
    if (!a.dgamma && !a.dbeta) return nullptr;
    if (a.chunks > 1) return a.parts + ((r * a.chunks + c) * 2 + which) * a.width;
    float* d = which ? a.dbeta : a.dgamma;
    return d ? d + r * a.grad_rank : nullptr;
}

// Bound by the bytes of x, dy and dx: 298 us at 8 x 4096 x 8192 bf16, 1.6 GB, 5.4 TB/s (and 67 MB of
// workgroups' sums, which take another 11 us to join); 36 us and 5 at 9 x 1001 x 2051 fp16, 111 MB (3.1 TB/s). With few rows the
// latency of a lane's rows one after another bounds it: 8.6 us at 81 x 16 tokens of 768 fp32.
template <typename T, int V, int LANES, int NV, bool STREAM>
__global__ __launch_bounds__(kBlock<LANES>, (kLocalGamma<V, LANES, NV> ? 4 : 1)) void norm_backward_kernel(Backward<T> a) {
    constexpr int G = kBlock<LANES> / LANES;
    __shared__ float2 slots[2][kWide / 64];
    __shared__ float join[G > 1 ? kThreads * NV * V : 1];
    const int lane = threadIdx.x % LANES, group = group_of_lane<LANES>();
    const Columns<V, LANES, NV> own(lane, (int)a.width);
    const float inv = 1.0f / (float)a.width;
    constexpr bool kLocal = kLocalGamma<V, LANES, NV>;
    __shared__ float gammas[kLocal ? LANES * NV * V : 1];
    float gamma[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        load_weights<V>(a.gamma, a.weight_type, own.first[j], a.width, 1.0f, gamma[j]);
    if constexpr (kLocal) {  // each lane reads only what it wrote
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) gammas[(j * LANES + lane) * V + k] = gamma[j][k];
    }
    int turn = 0;  // goes on from one rank to the next: no barrier stands between their rows
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t c = blockIdx.x, t1 = c * a.per;
        const int64_t t2 = t1 + a.per < a.tokens ? t1 + a.per : a.tokens;
        float dg[NV][V] = {}, db[NV][V] = {};
        struct Ahead {
            Some<T, V> x[NV], dy[NV];
            float mean, rstd;
        };
        const auto fetch = [&](int64_t t, Ahead& to) {
            const T* x = a.x + r * a.x_rank + t * a.x_token;
            const T* dy = a.dy + r * a.dy_rank + t * a.dy_token;
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (own.skip[j] < V) {
                    to.x[j] = load_vector<STREAM, V>(x + own.first[j]);
                    to.dy[j] = load_vector<STREAM, V>(dy + own.first[j]);
                }
            to.mean = a.mean[r * a.tokens + t];
            to.rstd = a.rstd[r * a.tokens + t];
        };
        // the next row is on its way during this row's sums, where there are registers for both
        constexpr bool kAhead = NV * V * sizeof(T) <= 64;
        const auto row = [&](int64_t t, Ahead& next) {
            if (!kAhead) fetch(t, next);
            float mean = next.mean, rstd = next.rstd;
            if constexpr (LANES >= 64) {  // the same in a wave: in scalar registers
                mean = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, mean)));
                rstd = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, rstd)));
            }
            float h[NV][V], g[NV][V];
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    h[j][k] = ((float)next.x[j][k] - mean) * rstd;
                    g[j][k] = (float)next.dy[j][k];
                    dg[j][k] += g[j][k] * h[j][k];
                    db[j][k] += g[j][k];
                    g[j][k] *= kLocal ? gammas[(j * LANES + lane) * V + k] : gamma[j][k];
                }
            if (kAhead && t + G < t2) fetch(t + G, next);
            float s1 = own.sum([&](int j, int k) { return g[j][k]; });
            float s2 = own.sum([&](int j, int k) { return g[j][k] * h[j][k]; });
            row_sums<LANES>(s1, s2, slots[turn]);
            turn ^= 1;
            s1 *= inv;
            s2 *= inv;
            T* dx = a.dx + r * a.dx_rank + t * a.dx_token;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                Some<T, V> o;
#pragma unroll
                for (int k = 0; k < V; ++k) o[k] = (T)(rstd * (g[j][k] - s1 - h[j][k] * s2));
                if (own.skip[j] < V) store_vector<STREAM, V>(dx + own.first[j], o);
            }
        };
        Ahead next;
        int64_t t = t1 + group;
        if (kAhead && t < t2) fetch(t, next);
        for (; t < t2; t += G) row(t, next);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float* out = sums_of(a, r, c, which);
            if (!out) continue;
            if constexpr (G == 1) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Some<float, V> o;
#pragma unroll
                    for (int k = 0; k < V; ++k) o[k] = which ? db[j][k] : dg[j][k];
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
                        if (own.skip[j] < V) join[group * N + own.first[j] + k] = which ? db[j][k] : dg[j][k];
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
}

// Rows beyond what a workgroup's registers hold: read twice, the second time from the caches, and the chunk's
// sums of the weight gradients added up where they go.
template <typename T>
__global__ __launch_bounds__(kWide) void norm_backward_long_kernel(Backward<T> a) {
    constexpr int V = kVec<T>;
    __shared__ float2 slots[2][kWide / 64];
    const float inv = 1.0f / (float)a.width;
    const int64_t i0 = (int64_t)threadIdx.x * V;
    int turn = 0;  // goes on from one rank to the next
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t c = blockIdx.x, t1 = c * a.per;
        const int64_t t2 = t1 + a.per < a.tokens ? t1 + a.per : a.tokens;
        float* dgamma = sums_of(a, r, c, 0);
        float* dbeta = sums_of(a, r, c, 1);
        // a lane adds to the same columns for every row
        for (int64_t i = i0; i < a.width; i += kWide * V) {
            const float zero[V] = {};
            if (dgamma) store_row<float, V>(dgamma, i, a.width, zero);
            if (dbeta) store_row<float, V>(dbeta, i, a.width, zero);
        }
        for (int64_t t = t1; t < t2; ++t) {
            const T* x = a.x + r * a.x_rank + t * a.x_token;
            const T* dy = a.dy + r * a.dy_rank + t * a.dy_token;
            T* dx = a.dx + r * a.dx_rank + t * a.dx_token;
            const float mean = a.mean[r * a.tokens + t], rstd = a.rstd[r * a.tokens + t];
            float h[V], g[V], gamma[V], s1 = 0.0f, s2 = 0.0f;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                load_row<T>(x, i, a.width, 0.0f, h);
                load_row<T>(dy, i, a.width, 0.0f, g);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    s1 += g[k] * gamma[k];
                    s2 += g[k] * gamma[k] * ((h[k] - mean) * rstd);
                }
            }
            row_sums<kWide>(s1, s2, slots[turn]);
            turn ^= 1;
            for (int64_t i = i0; i < a.width; i += kWide * V) {
                float o[V];
                load_row<T>(x, i, a.width, 0.0f, h);
                load_row<T>(dy, i, a.width, 0.0f, g);
                load_weights<V>(a.gamma, a.weight_type, i, a.width, 1.0f, gamma);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    h[k] = (h[k] - mean) * rstd;
                    o[k] = rstd * (g[k] * gamma[k] - s1 * inv - h[k] * (s2 * inv));
                }
                store_row<T, V>(dx, i, a.width, o);
                float s[V];
                if (dgamma) {
                    load_values<float, V>(dgamma, i, a.width, 0.0f, s);
#pragma unroll
                    for (int k = 0; k < V; ++k) s[k] += g[k] * h[k];
                    store_row<float, V>(dgamma, i, a.width, s);
                }
                if (dbeta) {
                    load_values<float, V>(dbeta, i, a.width, 0.0f, s);
#pragma unroll
                    for (int k = 0; k < V; ++k) s[k] += g[k];
                    store_row<float, V>(dbeta, i, a.width, s);
                }
            }
        }
    }
}

// The chunks' sums of every column of [sums][width], joined in the chunks' order by kJoinWaves waves of 64
// columns, in 64 bits. Eight loads of a wave are on their way: 11 us for 8 ranks of 128 chunks of 2 x 8192,
// 67 MB (6.2 TB/s).
constexpr int kJoinWaves = 8;

template <int SUMS>
__global__ __launch_bounds__(64 * kJoinWaves) void join_chunks_kernel(
    const float* parts, float* dgamma, float* dbeta, int64_t ranks, int64_t chunks, int64_t width,
    int64_t grad_rank) {
    __shared__ double sums[kJoinWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y) {
        double s = 0.0;
        if (col < SUMS * width) {
            const float* p = parts + r * chunks * SUMS * width + col;
#pragma unroll 8
            for (int64_t c = wave; c < chunks; c += kJoinWaves) s += p[c * SUMS * width];
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && col < SUMS * width) {
#pragma unroll
            for (int w = 1; w < kJoinWaves; ++w) s += sums[w][lane];
            float* out = col < width ? dgamma : dbeta;
            if (out) out[r * grad_rank + (col < width ? col : col - width)] = (float)s;
        }
        __syncthreads();
    }
}

// Workgroups of the forward pass: a few times what the GPU holds, with the same number of rows each, so that
// the weights are loaded once for all of them and a row's load overlaps the one before.
template <typename T>
int run_forward(Forward<T> a, hipStream_t stream) {
    if (a.x_rank == a.tokens * a.x_token && a.y_rank == a.tokens * a.y_token) {  // rank after rank
        a.tokens *= a.ranks;
        a.ranks = 1;
    }
    const Shape shape = shape_of<T>(a.width);
    const int64_t units = (a.tokens + group_rows(shape) - 1) / group_rows(shape);
    const int64_t most = imax(1, 256 * kBlocks * kThreads / block_lanes(shape) / a.ranks);
    const int64_t each = (units + most - 1) / most;
    const dim3 grid((unsigned)((units + each - 1) / each), (unsigned)imin(a.ranks, kMaxGridY));
#define RUN(V, L, N)                                                                      \
    if (a.stream) norm_forward_kernel<T, V, L, N, true><<<grid, kBlock<L>, 0, stream>>>(a); \
    else norm_forward_kernel<T, V, L, N, false><<<grid, kBlock<L>, 0, stream>>>(a)
#define RUN_LONG() norm_forward_long_kernel<T><<<grid, kWide, 0, stream>>>(a)
    TRIVANCE_NORM_SHAPES(RUN, RUN_LONG)
#undef RUN
#undef RUN_LONG
    return launch_status();
}

template <typename T>
int run_backward(const Backward<T>& a, hipStream_t stream) {
    const Shape shape = shape_of<T>(a.width);
    const dim3 grid((unsigned)a.chunks, (unsigned)imin(a.ranks, kMaxGridY));
#define RUN(V, L, N)                                                                       \
    if (a.stream) norm_backward_kernel<T, V, L, N, true><<<grid, kBlock<L>, 0, stream>>>(a); \
    else norm_backward_kernel<T, V, L, N, false><<<grid, kBlock<L>, 0, stream>>>(a)
#define RUN_LONG() norm_backward_long_kernel<T><<<grid, kWide, 0, stream>>>(a)
    TRIVANCE_NORM_SHAPES(RUN, RUN_LONG)
#undef RUN
#undef RUN_LONG
    const int rc = launch_status();
    if (rc || a.chunks == 1 || (!a.dgamma && !a.dbeta)) return rc;
    return join_chunks(a.parts, a.dgamma, a.dbeta, 2, a.ranks, a.chunks, a.width, a.grad_rank, stream);
}

}  // namespace

int join_chunks(const float* parts, float* dgamma, float* dbeta, int sums, int64_t ranks, int64_t chunks,
                int64_t width, int64_t grad_rank, hipStream_t stream) {
    const dim3 grid((unsigned)((sums * width + 63) / 64), (unsigned)imin(ranks, kMaxGridY));
    if (sums == 2)
        join_chunks_kernel<2><<<grid, 64 * kJoinWaves, 0, stream>>>(parts, dgamma, dbeta, ranks, chunks, width, grad_rank);
    else
        join_chunks_kernel<1><<<grid, 64 * kJoinWaves, 0, stream>>>(parts, dgamma, dbeta, ranks, chunks, width, grad_rank);
    return launch_status();
}

}  // namespace trivance

using namespace trivance;

extern "C" {

int trivance_layernorm_forward(const void* x, const void* gamma, const void* beta, void* y,
                               float* mean, float* rstd, int64_t ranks, int64_t tokens,
                               int64_t width, int64_t x_rank_stride, int64_t x_token_stride,
                               int64_t y_rank_stride, int64_t y_token_stride, double eps, int dtype,
                               int weight_dtype, void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype)) return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, width) || !(eps >= 0.0)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!x || !y || !rows_fit(ranks, tokens, width, x_rank_stride, x_token_stride) ||
        !rows_fit(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_distinct(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_in_place(y, x, ranks, tokens, y_rank_stride, y_token_stride, x_rank_stride, x_token_stride))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        return run_forward(Forward<T>{static_cast<const T*>(x), static_cast<T*>(y), gamma, beta, mean,
                                      rstd, ranks, tokens, width, x_rank_stride, x_token_stride,
                                      y_rank_stride, y_token_stride, (float)eps, weight_dtype,
                                      ranks * tokens * width * (int64_t)sizeof(T) > kStreamBytes},
                           s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

int64_t trivance_layernorm_workspace_bytes(int64_t ranks, int64_t tokens, int64_t width) {
    if (!sizes_ok(ranks, tokens, width)) return TRIVANCE_EINVAL;
    int64_t most = 0;
    for (const int dtype : {TRIVANCE_F32, TRIVANCE_BF16}) {
        const int64_t per = chunk_tokens(ranks, tokens, shape_of(width, dtype));
        const int64_t chunks = imax(1, (tokens + per - 1) / per);
        if (chunks > 1) most = imax(most, ranks * chunks * 2 * width * (int64_t)sizeof(float));
    }
    return most;
}

int trivance_layernorm_backward(const void* dy, const void* x, const void* gamma, const float* mean,
                                const float* rstd, void* dx, float* dgamma, float* dbeta,
                                int64_t ranks, int64_t tokens, int64_t width, int64_t dy_rank_stride,
                                int64_t dy_token_stride, int64_t x_rank_stride,
                                int64_t x_token_stride, int64_t dx_rank_stride,
                                int64_t dx_token_stride, int64_t grad_rank_stride, int dtype,
                                int weight_dtype, void* workspace, int64_t workspace_bytes,
                                void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype)) return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, width)) return TRIVANCE_EINVAL;
    if ((dgamma || dbeta) && !(rows_fit(ranks, 1, width, grad_rank_stride, 0) &&
                               rows_distinct(ranks, 1, width, grad_rank_stride, 0)))
        return TRIVANCE_EINVAL;
    if (tokens > 0 &&
        (!dy || !x || !mean || !rstd || !dx ||
         !rows_fit(ranks, tokens, width, dy_rank_stride, dy_token_stride) ||
         !rows_fit(ranks, tokens, width, x_rank_stride, x_token_stride) ||
         !rows_fit(ranks, tokens, width, dx_rank_stride, dx_token_stride) ||
         !rows_distinct(ranks, tokens, width, dx_rank_stride, dx_token_stride) ||
         !rows_in_place(dx, dy, ranks, tokens, dx_rank_stride, dx_token_stride, dy_rank_stride, dy_token_stride) ||
         !rows_in_place(dx, x, ranks, tokens, dx_rank_stride, dx_token_stride, x_rank_stride, x_token_stride)))
        return TRIVANCE_EINVAL;
    const int64_t need = trivance_layernorm_workspace_bytes(ranks, tokens, width);
    if ((dgamma || dbeta) && (workspace_bytes < need || (need > 0 && !workspace)))
        return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(float)) return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        const int64_t per = chunk_tokens(ranks, tokens, shape_of<T>(width));
        return run_backward(
            Backward<T>{static_cast<const T*>(dy), static_cast<const T*>(x), static_cast<T*>(dx), gamma,
                        mean, rstd, dgamma, dbeta, static_cast<float*>(workspace), ranks, tokens, width,
                        dy_rank_stride, dy_token_stride, x_rank_stride, x_token_stride, dx_rank_stride,
                        dx_token_stride, grad_rank_stride, imax(1, (tokens + per - 1) / per), per,
                        weight_dtype, ranks * tokens * width * (int64_t)sizeof(T) > kStreamBytes},
            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

}  // extern "C"
