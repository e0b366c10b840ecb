// What the operators around the AllReduce share: element types, rows of vectors that need not be
// aligned, sums over groups of lanes, and the checks of rows of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "trivance.h"

namespace trivance {

using f16 = _Float16;
using bf16 = __bf16;

// VEC consecutive values in 16 bytes. The type asks for no more alignment than an element's: the
// vector loads and stores of this GPU need none, so rows of any length and stride take the same path.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T>
struct Packed {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// Values i .. i + VEC of a row of `width` values as fp32; `fill` beyond the row's end.
template <typename T>
__device__ __forceinline__ void load_row(const T* row, int64_t i, int64_t width, float fill,
                                         float (&out)[kVec<T>]) {
    constexpr int V = kVec<T>;
    if (i + V <= width) {
        const typename Packed<T>::type x =
            *reinterpret_cast<const typename Packed<T>::type*>(row + i);
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = (float)x[k];
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = i + k < width ? (float)row[i + k] : fill;
    }
}

// V values of weights, whose type is known at run time (the branch is uniform and taken once a row
// or less); `fill` everywhere where there are none.
template <typename T, int V>
__device__ __forceinline__ void load_values(const void* p, int64_t i, int64_t width, float fill,
                                            float (&out)[V]) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    const T* row = static_cast<const T*>(p);
    if (i + V <= width) {
        const U x = *reinterpret_cast<const U*>(row + i);
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = (float)x[k];
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = i + k < width ? (float)row[i + k] : fill;
    }
}

template <int V>
__device__ __forceinline__ void load_weights(const void* p, int dtype, int64_t i, int64_t width,
                                             float fill, float (&out)[V]) {
    if (!p) {
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = fill;
    } else if (dtype == TRIVANCE_F32) {
        load_values<float, V>(p, i, width, fill, out);
    } else if (dtype == TRIVANCE_BF16) {
        load_values<bf16, V>(p, i, width, fill, out);
    } else {
        load_values<f16, V>(p, i, width, fill, out);
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_row(T* row, int64_t i, int64_t width, const float (&v)[V]) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (i + V <= width) {
        U x;
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = (T)v[k];
        *reinterpret_cast<U*>(row + i) = x;
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (i + k < width) row[i + k] = (T)v[k];
    }
}

// Sum and maximum over the L lanes (a power of two up to 64, aligned) that hold one row; every lane
// gets the result, the same bits in all of them.
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int d = 1; d < L; d *= 2) x += __shfl_xor(x, d);
    return x;
}

template <int L>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
    for (int d = 1; d < L; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

inline bool is_float_type(int dtype) {
    return dtype == TRIVANCE_F32 || dtype == TRIVANCE_BF16 || dtype == TRIVANCE_F16;
}

// Whether the strides of [ranks][tokens][width] rows address every value without overflow: neither
// is negative and the last element's index fits 62 bits. ranks, tokens, width >= 1.
inline bool rows_fit(int64_t ranks, int64_t tokens, int64_t width, int64_t rank_stride,
                     int64_t token_stride) {
    if (rank_stride < 0 || token_stride < 0) return false;
    const __int128 last = (__int128)(ranks - 1) * rank_stride + (__int128)(tokens - 1) * token_stride +
                          width;
    return last < ((__int128)1 << 60);
}

// Whether rows that are written do not share values: with more than one row, tokens are at least a
// row apart, and ranks at least a rank's tokens (or the other way round: tokens of different ranks
// interleaved).
inline bool rows_distinct(int64_t ranks, int64_t tokens, int64_t width, int64_t rank_stride,
                          int64_t token_stride) {
    if (tokens == 1) return ranks == 1 || rank_stride >= width;
    if (ranks == 1) return token_stride >= width;
    if (rank_stride >= token_stride)
        return token_stride >= width && rank_stride >= (tokens - 1) * token_stride + width;
    return rank_stride >= width && token_stride >= (ranks - 1) * rank_stride + width;
}

inline int launch_status() {
    return hipGetLastError() == hipSuccess ? TRIVANCE_OK : TRIVANCE_EHIP;
}

}  // namespace trivance
