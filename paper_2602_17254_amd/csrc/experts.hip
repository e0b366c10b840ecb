// Tokens sorted by expert and back, over the rows of [ranks][tokens][width].
//
//   the slots (token, j) of a rank that hold an expert, in the order of expert, token, j: slot i's place is p_i
//   dispatch:  rows_{p_tj} = x_t                      combine:  y_t = sum_j w_tj rows_{p_tj}
//   gradients: drows_{p_tj} = w_tj dy_t               dw_tj = sum over columns of dy_t rows_{p_tj}
//              of a dispatch: dx_t = sum_j drows_{p_tj}, a combine without weights
//
// Memory bounds all three. Every kernel goes by token: a token's row is read (or written) once and its slots' rows,
// which lie anywhere, in whole runs of consecutive lanes. A slot without a row (a place outside the sorted rows) is passed over: no sorted
// row is read or written for it. Its token's own row is read all the same, by the dispatch as its load goes before the places, by the
// gradient once for the token: with half of 8 x 8192 tokens of 2048 bf16 masked and a slot each they take 60 and 99 us, where 79 and
// 133 are those of all tokens and the bytes in use would take 40 and 59. Sums are in fp32, in the order of the slots, rounded once.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "device.h"
#include "operators.h"
#include "sort.h"
#include "strips.h"
#include "vectors.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

template <typename T>
struct Slots {
    const int* places;  // [ranks][tokens][top_k]
    const void* weights;  // the same, of weight_type; NULL: ones
    T* rows;            // the sorted rows, `capacity` of a rank
    int64_t ranks, tokens, width, capacity, rows_rank, rows_row;
    int64_t x_rank, x_token;  // of the tokens' rows
    int64_t drows_rank, drows_row;
    int top_k, weight_type;
    Share share;
};

// A slot's weight and its row's place, negative for none.
template <typename T>
__device__ __forceinline__ int place_of(const Slots<T>& a, int64_t slot) {
    const int p = a.places[slot];
    return p < a.capacity ? p : -1;
}

template <typename T>
__device__ __forceinline__ float weight_of(const Slots<T>& a, int64_t slot) {
    if (!a.weights) return 1.0f;
    if (a.weight_type == TRIVANCE_F32) return static_cast<const float*>(a.weights)[slot];
    if (a.weight_type == TRIVANCE_BF16) return (float)static_cast<const bf16*>(a.weights)[slot];
    return (float)static_cast<const f16*>(a.weights)[slot];
}

// A lane reads a vector of a token's row once and writes it to each of the token's slots' rows, one after another: 889 us for 8 x 16384
// tokens of 2048 bf16 in 8 slots, 4.8 GB (5.4 TB/s; 5.7 where the rows follow one another, 6.8 a copy). Stores to many rows bound
// it: all places first and then all stores took 955, a store a lane 1367 (latency), a wave for a row 965, fewer workgroups at
// once 898 to 957, contiguous tokens for each XCD 923.
template <typename T, int V, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void dispatch_kernel(Slots<T> a, const T* x) {
    for_vectors<V, 1>(a.share, a.ranks, a.tokens, a.width, [&](int64_t r, const Item(&item)[1]) {
        const auto v = load_vector<false, V>(x + r * a.x_rank + item[0].token * a.x_token + item[0].first);
        const int64_t slot = (r * a.tokens + item[0].token) * a.top_k;
        T* rows = a.rows + r * a.rows_rank + item[0].first;
        for (int j = 0; j < a.top_k; ++j) {
            const int p = place_of(a, slot + j);
            if (p >= 0) store_vector<STREAM, V>(rows + p * a.rows_row, v);
        }
    });
}

// A lane adds up vectors of U tokens' results, K slots at a time: all places, then all rows on their way at once. Bound by the bytes of the
// rows: 219 us for 8 x 8192 tokens of 2048 bf16 in 4 slots, 1.34 GB, 6.1 TB/s (248 with a slot's place and row one after
// the other, 226 with one token a lane); 20 us for 27 x 1003 tokens of 515 fp16 in 4 slots, half of them empty.
template <int K>
constexpr int kCombineItems = K <= 4 ? 2 : 1;

template <typename T, int V, int K, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void combine_kernel(Slots<T> a, T* y) {
    constexpr int U = kCombineItems<K>;
    for_vectors<V, U>(a.share, a.ranks, a.tokens, a.width, [&](int64_t r, const Item(&item)[U]) {
        const T* rows = a.rows + r * a.rows_rank;
        float sum[U][V] = {};
        for_strips<K>(0, a.top_k, [&](int j0, int here) {
            Some<T, V> v[U][K];
            int p[U][K];
            float w[U][K];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < K; ++j)
                    p[u][j] = item[u].is && j < here ? place_of(a, (r * a.tokens + item[u].token) * a.top_k + j0 + j) : -1;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (p[u][j] >= 0) {
                        v[u][j] = load_vector<STREAM, V>(rows + item[u].first + p[u][j] * a.rows_row);
                        w[u][j] = weight_of(a, (r * a.tokens + item[u].token) * a.top_k + j0 + j);
                    }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (p[u][j] >= 0) {
#pragma unroll
                        for (int k = 0; k < V; ++k) sum[u][k] += w[u][j] * (float)v[u][j][k];
                    }
        });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Some<T, V> o;
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = (T)sum[u][k];
            if (item[u].is) store_vector<STREAM, V>(y + r * a.x_rank + item[u].token * a.x_token + item[u].first, o);
        }
    });
}

// A product that is rounded to fp32 before it is to fewer bits, wherever it is stored: of some the compiler would make an
// instruction that rounds once, so that two lanes that write the same value might not.
__device__ __forceinline__ float product(float a, float b) {
    float p = a * b;
    asm("" : "+v"(p));
    return p;
}

// L lanes take a token: each adds up its vectors' part of the slots' sums, K slots at a time. With a workgroup for a token,
// whose lanes have a vector each or a few, 8 x 8192 tokens of 2048 bf16 in 4 slots take 427 us in place of a wave's 465.
template <typename T, int V, int L, int K, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void combine_backward_kernel(Slots<T> a, const T* dy, T* drows, float* dweights) {
    constexpr int G = kShareThreads / L;
    __shared__ float sums[L > 64 ? 2 : 1][L > 64 ? L / 64 : 1][K];
    int turn = 0;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        for (int64_t t = (int64_t)blockIdx.x * G + group; t < a.tokens; t += (int64_t)gridDim.x * G) {
            const int64_t slot = (r * a.tokens + t) * a.top_k;
            const T* from = dy + r * a.x_rank + t * a.x_token;
            for_strips<K>(0, a.top_k, [&](int j0, int here) {
                int p[K];
                float w[K], sum[K] = {};
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    p[j] = j < here ? place_of(a, slot + j0 + j) : -1;
                    w[j] = p[j] >= 0 ? weight_of(a, slot + j0 + j) : 0.0f;
                }
                for (int64_t i = lane * V; i < a.width; i += L * V) {
                    const int64_t at = i + V <= a.width ? i : a.width - V;
                    const int skip = (int)(i - at);  // values of the vector before
                    const auto d = load_vector<false, V>(from + at);
                    Some<T, V> v[K];
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (p[j] >= 0) v[j] = load_vector<STREAM, V>(a.rows + r * a.rows_rank + p[j] * a.rows_row + at);
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (p[j] >= 0) {
                            Some<T, V> o;
#pragma unroll
                            for (int k = 0; k < V; ++k) {
                                const float g = (float)d[k];
                                o[k] = (T)product(w[j], g);
                                sum[j] += k >= skip ? g * (float)v[j][k] : 0.0f;
                            }
                            T* to = drows + r * a.drows_rank + p[j] * a.drows_row + at;
                            if (skip == 0 || drows != a.rows) {
                                store_vector<STREAM, V>(to, o);
                            } else {  // in place: the wave of the vector before may not have read what is lent
#pragma unroll
                                for (int k = 1; k < V; ++k)
                                    if (k >= skip) to[k] = o[k];
                            }
                        }
                }
#pragma unroll
                for (int j = 0; j < K; ++j) sum[j] = lanes_sum<L < 64 ? L : 64>(sum[j]);
                if constexpr (L > 64) {
                    if (threadIdx.x % 64 == 0) {
#pragma unroll
                        for (int j = 0; j < K; ++j) sums[turn][threadIdx.x / 64][j] = sum[j];
                    }
                    __syncthreads();
                    if (lane < here) {
                        float s = 0.0f;
#pragma unroll
                        for (int w = 0; w < L / 64; ++w) s += sums[turn][w][lane];
                        dweights[slot + j0 + lane] = s;
                    }
                    turn ^= 1;
                } else if (lane == 0) {
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (j < here) dweights[slot + j0 + j] = sum[j];
                }
            });
        }
    }
}

template <typename F>
void with_slots(int64_t top_k, F run) {
    if (top_k == 1) run(std::integral_constant<int, 1>{});
    else if (top_k == 2) run(std::integral_constant<int, 2>{});
    else if (top_k <= 4) run(std::integral_constant<int, 4>{});
    else run(std::integral_constant<int, 8>{});
}

template <typename F>
int with_type(int dtype, F run) {
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

// Sizes that every call checks: all slots' numbers fit an int32.
bool sizes_ok(int64_t ranks, int64_t tokens, int64_t top_k) {
    if (ranks < 1 || tokens < 0 || top_k < 1) return false;
    return ranks <= INT32_MAX && top_k <= INT32_MAX && (__int128)ranks * tokens * top_k <= INT32_MAX;
}

// Whether the rows of tokens and the sorted ones can be addressed.
bool rows_ok(int64_t ranks, int64_t tokens, int64_t width, int64_t capacity, int64_t x_rank, int64_t x_token,
             int64_t rows_rank, int64_t rows_row) {
    if (width < 1 || width > ((int64_t)1 << 24) || capacity < 0 || capacity > INT32_MAX) return false;
    return rows_fit(ranks, tokens, width, x_rank, x_token) &&
           rows_fit(ranks, capacity > 0 ? capacity : 1, width, rows_rank, rows_row);
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" {

int64_t trivance_experts_workspace_bytes(int64_t ranks, int64_t tokens, int64_t top_k, int64_t experts) {
    if (!sizes_ok(ranks, tokens, top_k) || experts < 1) return TRIVANCE_EINVAL;
    if (experts > kMaxBins) return TRIVANCE_EUNSUPPORTED;
    return sort_hist_values(ranks, tokens * top_k, (int)experts) * (int64_t)sizeof(int);
}

int trivance_experts_sort(const void* chosen, const uint8_t* mask, int32_t* offsets, int32_t* places, int32_t* slots,
                          int64_t ranks, int64_t tokens, int64_t top_k, int64_t experts, int id_dtype, void* workspace,
                          int64_t workspace_bytes, void* stream) {
    if (id_dtype != TRIVANCE_I32 && id_dtype != TRIVANCE_I64) return TRIVANCE_EINVAL;
    const int64_t need = trivance_experts_workspace_bytes(ranks, tokens, top_k, experts);
    if (need < 0) return (int)need;
    if (!offsets || (tokens > 0 && (!chosen || !places))) return TRIVANCE_EINVAL;
    if (workspace_bytes < need || (need > 0 && !workspace)) return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(int)) return TRIVANCE_EINVAL;
    SortPass a{};
    a.ids = tokens > 0 ? chosen : offsets;  // of no tokens nothing is read
    a.mask = mask;
    a.wide = id_dtype == TRIVANCE_I64;
    a.by_top_k = make_fastdiv32((uint32_t)top_k);
    a.tokens = tokens;
    a.ranks = ranks;
    a.slots = tokens * top_k;
    a.bound = experts;
    a.digits = -1;
    a.bins = (int)experts;
    a.places = places;
    a.offsets = offsets;
    a.to_order = slots;
    a.hist = static_cast<int*>(workspace);
    return run_sort_pass(a, reinterpret_cast<hipStream_t>(stream));
}

int trivance_experts_dispatch(const void* x, const int32_t* places, void* rows, int64_t ranks, int64_t tokens,
                              int64_t top_k, int64_t width, int64_t capacity, int64_t x_rank_stride,
                              int64_t x_token_stride, int64_t rows_rank_stride, int64_t rows_row_stride, int dtype,
                              void* stream) {
    if (!is_float_type(dtype) || !sizes_ok(ranks, tokens, top_k)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!rows_ok(ranks, tokens, width, capacity, x_rank_stride, x_token_stride, rows_rank_stride, rows_row_stride))
        return TRIVANCE_EINVAL;
    if (!x || !places || (capacity > 0 && !rows) || rows == x ||
        (capacity > 0 && !rows_distinct(ranks, capacity, width, rows_rank_stride, rows_row_stride)))
        return TRIVANCE_EINVAL;
    if (capacity == 0) return TRIVANCE_OK;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_vector<T>(width, [&](auto v) {
            Slots<T> a{places, nullptr, static_cast<T*>(rows), ranks, tokens, width, capacity, rows_rank_stride,
                       rows_row_stride, x_rank_stride, x_token_stride, 0, 0, (int)top_k, 0,
                       share_vectors(ranks, tokens, width, v(), 1, false)};
            const T* from = static_cast<const T*>(x);
            if (ranks * tokens * top_k * width * (int64_t)sizeof(T) > kStreamBytes)
                dispatch_kernel<T, v(), true><<<a.share.grid, kShareThreads, 0, s>>>(a, from);
            else
                dispatch_kernel<T, v(), false><<<a.share.grid, kShareThreads, 0, s>>>(a, from);
            return launch_status();
        });
    });
}

int trivance_experts_combine(const void* rows, const int32_t* places, const void* weights, void* y, int64_t ranks,
                             int64_t tokens, int64_t top_k, int64_t width, int64_t capacity, int64_t rows_rank_stride,
                             int64_t rows_row_stride, int64_t y_rank_stride, int64_t y_token_stride, int dtype,
                             int weight_dtype, void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype) || !sizes_ok(ranks, tokens, top_k)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!rows_ok(ranks, tokens, width, capacity, y_rank_stride, y_token_stride, rows_rank_stride, rows_row_stride))
        return TRIVANCE_EINVAL;
    if ((capacity > 0 && !rows) || !places || !y || y == rows ||
        !rows_distinct(ranks, tokens, width, y_rank_stride, y_token_stride))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_vector<T>(width, [&](auto v) {
            Slots<T> a{places, weights, static_cast<T*>(const_cast<void*>(rows)), ranks, tokens, width, capacity,
                       rows_rank_stride, rows_row_stride, y_rank_stride, y_token_stride, 0, 0, (int)top_k, weight_dtype, Share{}};
            with_slots(top_k, [&](auto k) {
                a.share = share_vectors(ranks, tokens, width, v(), kCombineItems<k()>, false);
                if (ranks * tokens * top_k * width * (int64_t)sizeof(T) > kStreamBytes)
                    combine_kernel<T, v(), k(), true><<<a.share.grid, kShareThreads, 0, s>>>(a, static_cast<T*>(y));
                else
                    combine_kernel<T, v(), k(), false><<<a.share.grid, kShareThreads, 0, s>>>(a, static_cast<T*>(y));
            });
            return launch_status();
        });
    });
}

int trivance_experts_combine_backward(const void* dy, const void* rows, const int32_t* places, const void* weights,
                                      void* drows, float* dweights, int64_t ranks, int64_t tokens, int64_t top_k,
                                      int64_t width, int64_t capacity, int64_t dy_rank_stride, int64_t dy_token_stride,
                                      int64_t rows_rank_stride, int64_t rows_row_stride, int64_t drows_rank_stride,
                                      int64_t drows_row_stride, int dtype, int weight_dtype, void* stream) {
    if (!is_float_type(dtype) || !is_float_type(weight_dtype) || !sizes_ok(ranks, tokens, top_k)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!rows_ok(ranks, tokens, width, capacity, dy_rank_stride, dy_token_stride, rows_rank_stride, rows_row_stride))
        return TRIVANCE_EINVAL;
    if (!dy || !places || !dweights || drows == dy || (capacity > 0 && (!rows || !drows)) ||
        !rows_fit(ranks, capacity > 0 ? capacity : 1, width, drows_rank_stride, drows_row_stride) ||
        (capacity > 0 &&
         (!rows_distinct(ranks, capacity, width, drows_rank_stride, drows_row_stride) ||
          !rows_in_place(drows, rows, ranks, capacity, drows_rank_stride, drows_row_stride, rows_rank_stride, rows_row_stride))))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_vector<T>(width, [&](auto v) {
            const Slots<T> a{places, weights, static_cast<T*>(const_cast<void*>(rows)), ranks, tokens, width, capacity,
                             rows_rank_stride, rows_row_stride, dy_rank_stride, dy_token_stride, drows_rank_stride,
                             drows_row_stride, (int)top_k, weight_dtype, Share{}};
            const T* from = static_cast<const T*>(dy);
            const bool stream_rows = ranks * tokens * top_k * width * (int64_t)sizeof(T) > kStreamBytes;
            const auto launch = [&](auto l, auto k) {
                const dim3 grid = share_rows(ranks, tokens, kShareThreads / l());
                if (stream_rows)
                    combine_backward_kernel<T, v(), l(), k(), true><<<grid, kShareThreads, 0, s>>>(
                        a, from, static_cast<T*>(drows), dweights);
                else
                    combine_backward_kernel<T, v(), l(), k(), false><<<grid, kShareThreads, 0, s>>>(
                        a, from, static_cast<T*>(drows), dweights);
            };
            with_slots(top_k, [&](auto k) {
                // lanes of a token: a power of two that holds its vectors, or a wave; the workgroup for more than two of a wave's
                const int64_t n = (width + v() - 1) / v();
                if (n <= 8) launch(std::integral_constant<int, 8>{}, k);
                else if (n <= 16) launch(std::integral_constant<int, 16>{}, k);
                else if (n <= 32) launch(std::integral_constant<int, 32>{}, k);
                else if (n <= 128) launch(std::integral_constant<int, 64>{}, k);
                else launch(std::integral_constant<int, 256>{}, k);
            });
            return launch_status();
        });
    });
}

}  // extern "C"
