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

// V of them.
template <typename T, int V>
using Some = T __attribute__((ext_vector_type(V), aligned(sizeof(T))));

// A vector load or store that, where STREAM, does not stay in the caches: of tensors beyond kStreamBytes,
// the L2 caches together, which would drop it before its next reader.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

template <bool STREAM, int V, typename T>
__device__ __forceinline__ auto load_vector(const T* p) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const U*>(p));
    else return *reinterpret_cast<const U*>(p);
}

template <bool STREAM, int V, typename T, typename U>
__device__ __forceinline__ void store_vector(T* p, U v) {
    typedef T W __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<W*>(p));
    else *reinterpret_cast<W*>(p) = v;
}

// A lane's vector of a row as it lies in memory, values i .. i + VEC; `fill` beyond the row's end.
template <typename T, bool STREAM = false>
__device__ __forceinline__ typename Packed<T>::type load_packed(const T* row, int64_t i, int64_t width, T fill) {
    constexpr int V = kVec<T>;
    typename Packed<T>::type x;
    if (i + V <= width) {
        x = load_vector<STREAM, V>(row + i);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = fill;
        if (i < width) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (i + k < width) x[k] = row[i + k];
        }
    }
    return x;
}

// The same as fp32.
template <typename T>
__device__ __forceinline__ void load_row(const T* row, int64_t i, int64_t width, float fill,
                                         float (&out)[kVec<T>]) {
    const typename Packed<T>::type x = load_packed<T>(row, i, width, (T)fill);
#pragma unroll
    for (int k = 0; k < kVec<T>; ++k) out[k] = (float)x[k];
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

template <typename T, int V, bool STREAM = false>
__device__ __forceinline__ void store_row(T* row, int64_t i, int64_t width, const float (&v)[V]) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (i + V <= width) {
        U x;
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = (T)v[k];
        store_vector<STREAM, V>(row + i, x);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (i + k < width) row[i + k] = (T)v[k];
    }
}

// Sum and maximum over the L lanes (a power of two up to 64, aligned) that hold one row; every lane
// gets the result, the same bits in all of them. The partner of a step differs in one bit of the lane up to
// 2; then mirroring 8 and 16 lanes and exchanging halves of 32 and 64 bring together what
// the steps before have made equal. One instruction a step, and none of local memory's latency.
template <int CONTROL>
__device__ __forceinline__ int word_from_lane(int x) {
    return __builtin_amdgcn_mov_dpp(x, CONTROL, 0xf, 0xf, true);
}

template <int CONTROL>
__device__ __forceinline__ float from_lane(float x) {
    return __builtin_bit_cast(float, word_from_lane<CONTROL>(__builtin_bit_cast(int, x)));
}

struct Words {
    int lo, hi;
};

template <int CONTROL>
__device__ __forceinline__ double from_lane(double x) {
    const Words w = __builtin_bit_cast(Words, x);
    return __builtin_bit_cast(double, Words{word_from_lane<CONTROL>(w.lo), word_from_lane<CONTROL>(w.hi)});
}

// v_permlaneN_swap exchanges the odd rows of N lanes of its first register with the even rows of its
// second: of two copies, each lane then holds the pair's values. (The builtins of this compiler
// return the first register for both; two wait states stand between the copies and the exchange.)
template <int N>
__device__ __forceinline__ void exchange(int& x, int& y) {
    if constexpr (N == 16) asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    else asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
}

template <int N, typename OP>
__device__ __forceinline__ float with_pair(float x, OP op) {
    int a = __builtin_bit_cast(int, x), b = a;
    exchange<N>(a, b);
    return op(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

template <int N, typename OP>
__device__ __forceinline__ double with_pair(double x, OP op) {
    Words a = __builtin_bit_cast(Words, x), b = a;
    exchange<N>(a.lo, b.lo);
    exchange<N>(a.hi, b.hi);
    return op(__builtin_bit_cast(double, a), __builtin_bit_cast(double, b));
}

template <int L, typename F, typename OP>
__device__ __forceinline__ F over_lanes(F x, OP op) {
    if constexpr (L >= 2) x = op(x, from_lane<0xB1>(x));    // quads 1 0 3 2
    if constexpr (L >= 4) x = op(x, from_lane<0x4E>(x));    // quads 2 3 0 1
    if constexpr (L >= 8) x = op(x, from_lane<0x141>(x));   // halves of 16 mirrored
    if constexpr (L >= 16) x = op(x, from_lane<0x140>(x));  // 16 mirrored
    if constexpr (L >= 32) x = with_pair<16>(x, op);
    if constexpr (L >= 64) x = with_pair<32>(x, op);
    return x;
}

template <int L, typename F>
__device__ __forceinline__ F lanes_sum(F x) {
    return over_lanes<L>(x, [](F a, F b) { return a + b; });
}

template <int L>
__device__ __forceinline__ float lanes_max(float x) {
    return over_lanes<L>(x, [](float a, float b) { return fmaxf(a, b); });
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

// Whether rows that are written may lie where rows that are read do: elsewhere, or each in its own place. With other
// strides they would overwrite rows that are still to be read. Strides of a single rank or token do not matter.
inline bool rows_in_place(const void* out, const void* in, int64_t ranks, int64_t tokens, int64_t out_rank_stride,
                          int64_t out_token_stride, int64_t in_rank_stride, int64_t in_token_stride) {
    return out != in || ((ranks == 1 || out_rank_stride == in_rank_stride) &&
                         (tokens == 1 || out_token_stride == in_token_stride));
}

inline int launch_status() {
    return hipGetLastError() == hipSuccess ? TRIVANCE_OK : TRIVANCE_EHIP;
}

}  // namespace trivance
