// Dropout of [ranks][tokens][width] rows with a mask that is never stored.
//
//   y = residual + keep x / (1 - q),     q = limit / 65536,     keep where the value's 16 random bits >= limit
//
// The bits come from Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw 2011): the key is the seed, the counter
// (column / 8, token, rank, call). A block of 128 bits serves the eight columns, the low half of each word first,
// so a value's bits depend on its place alone, not on strides, types, the launch or the number of ranks; the gradient is
// the same call on dy. Seed and call number lie in device memory: a captured graph draws new masks as
// the program counts the call up.
// Memory bounds it, the generator being close behind: ten rounds take 20 products of 64 bits and some 40 other
// operations for eight values. With 32 bits a value it would take twice that. 8 x 4096 x 8192 bf16 with a residual 266 us, 1.6 GB, 6.0 TB/s.
// Rows that end inside a block cost more, as their last values are stored one by one: 8 x 8192 x 1500 81 us, 4.8 TB/s.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "operators.h"
#include "vectors.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

constexpr int kBlock = 8;  // columns of a counter

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)c[0] * 0xD2511F53u, q = (uint64_t)c[2] * 0xCD9E8D57u;
        const uint32_t c0 = (uint32_t)(q >> 32) ^ c[1] ^ k0, c2 = (uint32_t)(p >> 32) ^ c[3] ^ k1;
        c[1] = (uint32_t)q;
        c[3] = (uint32_t)p;
        c[0] = c0;
        c[2] = c2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

template <typename T>
struct Dropout {
    const T *x, *residual;
    T* y;
    const uint64_t* state;  // seed, call
    int64_t ranks, tokens, width, x_rank, x_token, residual_rank, residual_token, y_rank, y_token;
    uint32_t limit;
    float scale;
    Share share;
};

template <typename T, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void dropout_kernel(Dropout<T> a) {
    constexpr int V = kVec<T>, N = kBlock / V;
    const uint64_t seed = a.state[0];
    const uint32_t call = (uint32_t)a.state[1];
    // no lent values: a block's columns are those of its counter, and y may be x
    for_vectors<kBlock, 1>(a.share, a.ranks, a.tokens, INT64_MAX, [&](int64_t r, const Item(&item)[1]) {
        const int64_t t = item[0].token, first = item[0].first;
        const T* x = a.x + r * a.x_rank + t * a.x_token;
        const T* residual = a.residual + r * a.residual_rank + t * a.residual_token;
        T* y = a.y + r * a.y_rank + t * a.y_token;
        typename Packed<T>::type v[N], more[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = load_columns<T, STREAM>(x, first + n * V, a.width);
            if (a.residual) more[n] = load_columns<T, STREAM>(residual, first + n * V, a.width);
        }
        uint32_t c[4] = {(uint32_t)(first / kBlock), (uint32_t)t, (uint32_t)r, call};
        philox(c, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float o[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int i = n * V + k;
                const uint32_t bits = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xFFFFu;
                o[k] = bits >= a.limit ? (float)v[n][k] * a.scale : 0.0f;
                if (a.residual) o[k] += (float)more[n][k];
            }
            store_row<T, V, STREAM>(y, first + n * V, a.width, o);
        }
    });
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" int trivance_dropout(const void* x, const void* residual, void* y, const uint64_t* state, int64_t ranks,
                                int64_t tokens, int64_t width, int64_t x_rank_stride, int64_t x_token_stride,
                                int64_t residual_rank_stride, int64_t residual_token_stride, int64_t y_rank_stride,
                                int64_t y_token_stride, double rate, int dtype, void* stream) {
    if (!is_float_type(dtype) || !(rate >= 0.0 && rate <= 1.0)) return TRIVANCE_EINVAL;
    const uint32_t limit = (uint32_t)__builtin_rint(rate * 65536.0);
    if (limit > 65535) return TRIVANCE_EINVAL;
    if (ranks < 1 || tokens < 0 || width < 1 || width > ((int64_t)1 << 24) || ranks > UINT32_MAX || tokens > UINT32_MAX)
        return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!x || !y || !state || reinterpret_cast<uintptr_t>(state) % sizeof(uint64_t) ||
        !rows_fit(ranks, tokens, width, x_rank_stride, x_token_stride) ||
        !rows_fit(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_distinct(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_in_place(y, x, ranks, tokens, y_rank_stride, y_token_stride, x_rank_stride, x_token_stride) ||
        (residual && (!rows_fit(ranks, tokens, width, residual_rank_stride, residual_token_stride) ||
                      !rows_in_place(y, residual, ranks, tokens, y_rank_stride, y_token_stride, residual_rank_stride,
                                     residual_token_stride))))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        const Dropout<T> a{static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(y), state, ranks,
                           tokens, width, x_rank_stride, x_token_stride, residual_rank_stride, residual_token_stride,
                           y_rank_stride, y_token_stride, limit, (float)(65536.0 / (65536.0 - limit)),
                           share_vectors(ranks, tokens, width, kBlock, 1, true)};
        if ((double)ranks * tokens * width * sizeof(T) > kStreamBytes)
            dropout_kernel<T, true><<<a.share.grid, kShareThreads, 0, s>>>(a);
        else
            dropout_kernel<T, false><<<a.share.grid, kShareThreads, 0, s>>>(a);
        return launch_status();
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}
