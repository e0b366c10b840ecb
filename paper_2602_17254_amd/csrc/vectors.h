// Kernels that take the vectors of [ranks][tokens][width] rows one by one: how they are shared out to lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "device.h"
#include "operators.h"

namespace trivance {

constexpr int kShareThreads = 256;
constexpr int64_t kShareMaxY = 65535;
constexpr int64_t kShareMaxX = (int64_t)1 << 22;  // 2^30 lanes of a launch at most

// A workgroup takes the vectors of `tokens` consecutive tokens of a rank.
struct Share {
    uint32_t vectors;  // of a row
    FastDiv32 by_vectors;
    uint32_t tokens;
    dim3 grid;
};

// As many tokens as the lanes hold with `times` vectors each, one at least. With `fill`, where there are workgroups enough, up to four
// times as many, if fewer lanes are then without a vector in the last round: 188 vectors are 73% of 256 lanes' work, four
// times 188 are 98% of three rounds.
inline Share share_vectors(int64_t ranks, int64_t tokens, int64_t width, int vec, int times, bool fill) {
    const int64_t n = (width + vec - 1) / vec, lanes = (int64_t)kShareThreads * times;  // n below 2^24
    const int64_t fit = n < lanes ? lanes / n : 1;
    const auto rounds = [&](int64_t tokens) { return (tokens * n + lanes - 1) / lanes; };
    int64_t each = fit;
    for (int64_t e = fit + 1; fill && e <= 4 * fit; ++e)
        if ((double)ranks * tokens / e >= 4096 && 100 * rounds(e) * each < 95 * rounds(each) * e) each = e;
    const int64_t blocks = (tokens + each - 1) / each;
    return Share{(uint32_t)n, make_fastdiv32((uint32_t)n), (uint32_t)each,
                 dim3((unsigned)(blocks < kShareMaxX ? blocks : kShareMaxX), (unsigned)(ranks < kShareMaxY ? ranks : kShareMaxY))};
}

// Workgroups that take `rows` tokens at a time.
inline dim3 share_rows(int64_t ranks, int64_t tokens, int64_t rows) {
    const int64_t blocks = (tokens + rows - 1) / rows;
    return dim3((unsigned)(blocks < kShareMaxX ? blocks : kShareMaxX), (unsigned)(ranks < kShareMaxY ? ranks : kShareMaxY));
}

// One of the vectors that a lane takes at once.
struct Item {
    bool is;  // whether there is one
    int64_t token;
    int64_t first;  // of its columns
};

// run(rank, items) for every vector of every row, U of them at once. A row that does not end with a vector of V values
// lends its last one values of the one before: both write the same there. V is 1 for rows shorter than a vector.
template <int V, int U, typename F>
__device__ __forceinline__ void for_vectors(const Share& s, int64_t ranks, int64_t tokens, int64_t width, F run) {
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y)
        for (int64_t t0 = (int64_t)blockIdx.x * s.tokens; t0 < tokens; t0 += (int64_t)gridDim.x * s.tokens) {
            const uint32_t here = (tokens - t0 < s.tokens ? (uint32_t)(tokens - t0) : s.tokens) * s.vectors;
            for (uint32_t i0 = threadIdx.x; i0 < here; i0 += U * kShareThreads) {
                Item item[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t i = i0 + u * kShareThreads, of = fdiv32(i, s.by_vectors);
                    const int64_t first = (int64_t)(i - of * s.vectors) * V;
                    item[u] = Item{i < here, t0 + of, first + V <= width ? first : width - V};
                }
                run(r, item);
            }
        }
}

// A vector of a row where nothing may be lent, as y may be x: what lies behind the row's end is not read, and what
// the result holds there does not matter. A row's last values come by single loads, all on their way at once.
template <typename T, bool STREAM>
__device__ __forceinline__ typename Packed<T>::type load_columns(const T* row, int64_t i, int64_t width) {
    constexpr int V = kVec<T>;
    typename Packed<T>::type x = {};
    if (i + V <= width) {
        x = load_vector<STREAM, V>(row + i);
    } else if (i < width) {
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = row[i + k < width ? i + k : width - 1];
    }
    return x;
}

// run with the number of values of a row's vectors.
template <typename T, typename F>
int with_vector(int64_t width, F run) {
    if (width < kVec<T>) return run(std::integral_constant<int, 1>{});
    return run(std::integral_constant<int, kVec<T>>{});
}

}  // namespace trivance
