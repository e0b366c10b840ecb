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

// A workgroup takes the vectors of `tokens` consecutive tokens of a rank: as many as its lanes hold, one at least.
struct Share {
    uint32_t vectors;  // of a row
    FastDiv32 by_vectors;
    uint32_t tokens;
    dim3 grid;
};

inline Share share_vectors(int64_t ranks, int64_t tokens, int64_t width, int vec) {
    const int64_t n = (width + vec - 1) / vec;  // below 2^24
    const int64_t each = n < kShareThreads ? kShareThreads / n : 1, blocks = (tokens + each - 1) / each;
    return Share{(uint32_t)n, make_fastdiv32((uint32_t)n), (uint32_t)each,
                 dim3((unsigned)(blocks < kShareMaxX ? blocks : kShareMaxX), (unsigned)(ranks < kShareMaxY ? ranks : kShareMaxY))};
}

// Workgroups that take `rows` tokens at a time.
inline dim3 share_rows(int64_t ranks, int64_t tokens, int64_t rows) {
    const int64_t blocks = (tokens + rows - 1) / rows;
    return dim3((unsigned)(blocks < kShareMaxX ? blocks : kShareMaxX), (unsigned)(ranks < kShareMaxY ? ranks : kShareMaxY));
}

// run(rank, token, vector) for every vector of every row.
template <typename F>
__device__ __forceinline__ void for_blocks(const Share& s, int64_t ranks, int64_t tokens, F run) {
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y)
        for (int64_t t0 = (int64_t)blockIdx.x * s.tokens; t0 < tokens; t0 += (int64_t)gridDim.x * s.tokens) {
            const uint32_t here = tokens - t0 < s.tokens ? (uint32_t)(tokens - t0) : s.tokens;
            for (uint32_t i = threadIdx.x; i < here * s.vectors; i += kShareThreads) {
                const uint32_t of = fdiv32(i, s.by_vectors);
                run(r, t0 + of, i - of * s.vectors);
            }
        }
}

// run(rank, token, first column) for every vector of V values. A row that does not end with a vector lends its last one
// values of the one before: both write the same there. V is 1 for rows shorter than a vector.
template <int V, typename F>
__device__ __forceinline__ void for_vectors(const Share& s, int64_t ranks, int64_t tokens, int64_t width, F run) {
    for_blocks(s, ranks, tokens, [&](int64_t r, int64_t t, uint32_t vector) {
        const int64_t first = (int64_t)vector * V;
        run(r, t, first + V <= width ? first : width - V);
    });
}

// run with the number of values of a row's vectors.
template <typename T, typename F>
int with_vector(int64_t width, F run) {
    if (width < kVec<T>) return run(std::integral_constant<int, 1>{});
    return run(std::integral_constant<int, kVec<T>>{});
}

}  // namespace trivance
