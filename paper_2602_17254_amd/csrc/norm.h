// What the norms over rows of [ranks][tokens][width] share: how a row lies in the registers of a group of
// lanes, sums over it, how a rank's tokens are shared out to workgroups, and the join of the workgroups' sums
// of weight gradients.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "operators.h"

// the norms' products and sums are fused, those in the functions here among them
#pragma clang fp contract(fast)

namespace trivance {

constexpr int kThreads = 256;      // lanes of a workgroup whose rows take fewer
constexpr int kWide = 1024;        // lanes of the widest rows' groups
constexpr int64_t kMaxGridY = 65535;

template <int LANES>
constexpr int kBlock = LANES < kThreads ? kThreads : LANES;

// Sum over the LANES lanes that hold a row. Rows wider than a wave meet in local memory, in `slot`,
// which alternates between two from one sum to the next: the barrier of the second sum stands between
// the reads of the first and the writes of the third.
template <int LANES, typename F>
__device__ __forceinline__ F row_sum(F x, F* slot) {
    if constexpr (LANES <= 64) return lanes_sum<LANES>(x);
    constexpr int kWaves = LANES / 64;
    x = lanes_sum<64>(x);
    if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = x;
    __syncthreads();
    F s = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += slot[w];
    return s;
}

// Both row sums of the backward pass with one barrier; `slots` alternate from each row of a workgroup to its next,
// whatever their ranks: a row's barrier stands between the reads of the row before it and the writes of
// the row after it.
template <int LANES>
__device__ __forceinline__ void row_sums(float& x, float& y, float2* slots) {
    x = lanes_sum<LANES <= 64 ? LANES : 64>(x);
    y = lanes_sum<LANES <= 64 ? LANES : 64>(y);
    if constexpr (LANES > 64) {
        if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = make_float2(x, y);
        __syncthreads();
        x = y = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) {
            const float2 s = slots[w];
            x += s.x;
            y += s.y;
        }
    }
}

// A lane's part of every row: NV vectors of V values, one every LANES vectors. Rows that do not end with a
// vector lend the last lane values of the one before: it reads and writes them as well, the same bits,
// and leaves them out of its sums. So a row needs no path for its end; rows shorter than a vector
// take V = 1.
template <int V, int LANES, int NV>
struct Columns {
    int first[NV];  // of the lane's values
    int skip[NV];   // those that count for another lane; V: the lane has none
    __device__ __forceinline__ Columns(int lane, int width) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = (j * LANES + lane) * V;
            first[j] = i + V <= width ? i : width - V;
            skip[j] = i < width ? i - first[j] : V;
        }
    }
    // The sum of f(j, k), of its type, over the values that count.
    template <typename F>
    __device__ __forceinline__ auto sum(F f) const {
        decltype(f(0, 0)) s = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            decltype(f(0, 0)) part = 0;
            if (skip[j] == 0) {
#pragma unroll
                for (int k = 0; k < V; ++k) part += f(j, k);
            } else {
                // few lanes come here: without the barrier to the compiler, it works out the V
                // comparisons before a kernel's loop and has no registers left for them
                int from = skip[j];
                asm volatile("" : "+v"(from));
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (k >= from) part += f(j, k);
            }
            s += part;
        }
        return s;
    }
};

// The group of lanes of a row: known to be the same in a whole wave where a row takes one or more.
template <int LANES>
__device__ __forceinline__ int group_of_lane() {
    if constexpr (LANES > 64) return 0;
    const int g = threadIdx.x / LANES;
    if constexpr (LANES == 64) return __builtin_amdgcn_readfirstlane(g);
    return g;
}

// Whether gamma stays in local memory, so that the registers suffice for two workgroups of 512 lanes on a CU, or four of
// 256: some go on while others wait for their row's sums. With 256 lanes 2 x 8192 x 2200 bf16 takes 57 us in place of
// 66, 8 x 4096 x 2048 85 in place of 104, 8 x 4096 x 4096 161 in place of 166; sizes whose workgroups have
// a few rows each lose up to 2%, as 4 x 500 x 4000 fp16 (20.8 in place of 20.4) and 16 x 128 x 1536 bf16
// (14.0 in place of 13.8).
template <int V, int LANES, int NV>
constexpr bool kLocalGamma = (LANES == 256 || LANES == 512) && V == 8 && NV == 2;

// How a row lies in lanes: groups of 8 to 64 lanes with one vector each, then waves and larger groups
// with 16 values a lane; 32 for the widest, whose workgroups would need more registers with 1024 lanes
// than those have. kTiny: shorter than a vector; kLong: in no workgroup's registers.
enum class Shape { kTiny, k8, k16, k32, k64, k64x2, k64x4, k256x2, k256x4, k512x2, k512x4, k512x8, kLong };

template <typename T>
Shape shape_of(int64_t width) {
    constexpr int V = kVec<T>;
    const int64_t n = (width + V - 1) / V;
    if (width < V) return Shape::kTiny;
    if (n <= 8) return Shape::k8;
    if (n <= 16) return Shape::k16;
    if (n <= 32) return Shape::k32;
    if (n <= 64) return Shape::k64;
    if (n <= 128) return Shape::k64x2;
    if (V == 4) {
        if (n <= 256) return Shape::k64x4;
        if (n <= 512) return Shape::k256x2;
        if (n <= 1024) return Shape::k256x4;
        if (n <= 2048) return Shape::k512x4;
        if (n <= 4096) return Shape::k512x8;
        return Shape::kLong;
    }
    if (n <= 512) return Shape::k256x2;
    if (n <= 1024) return Shape::k512x2;
    if (n <= 2048) return Shape::k512x4;
    return Shape::kLong;
}

// The rows that a workgroup takes at a time, and its lanes.
inline int group_rows(Shape s) {
    switch (s) {
        case Shape::kTiny: case Shape::k8: return kThreads / 8;
        case Shape::k16: return kThreads / 16;
        case Shape::k32: return kThreads / 32;
        case Shape::k64: case Shape::k64x2: case Shape::k64x4: return kThreads / 64;
        default: return 1;
    }
}

inline int block_lanes(Shape s) {
    switch (s) {
        case Shape::k512x2: case Shape::k512x4: case Shape::k512x8: return 512;
        case Shape::kLong: return kWide;
        default: return kThreads;
    }
}

inline int64_t imin(int64_t a, int64_t b) { return a < b ? a : b; }
inline int64_t imax(int64_t a, int64_t b) { return a > b ? a : b; }

// The tokens that a chunk of the backward pass takes. Two workgroups a CU (512; one where a row takes 512
// lanes), of four rows at least for each group of lanes, so that few tokens still spread over the GPU;
// four a CU where each then has 16 rows or more, as each chunk's sums take a way through memory. With 8 rows
// enough for that, 19 sizes between the two took 2% more in all: 8 x 1200 x 16000 bf16 262 us in place of 219,
// 8 x 5000 x 768 bf16 51 in place of 44, 1 x 9000 x 4000 bf16 59 in place of 54; 1 x 16000 x 1100 bf16 46 in
// place of 54 and 8 x 1500 x 1536 bf16 35 in place of 39, whose lanes' second vectors are void. A few
// workgroups above a multiple of what the CUs hold would cost a round. All these are the layer norm's times; the RMS
// norm's backward pass follows the same rule, which was not measured against others for it.
inline int64_t chunk_tokens(int64_t ranks, int64_t tokens, Shape s) {
    const int64_t rows = group_rows(s), wide = block_lanes(s) / kThreads;
    const int64_t many = imax(1, 1024 / ranks), few = imax(1, 512 / wide / ranks);
    const int64_t chunks = imax(1, many * 16 * rows <= tokens ? many : imin(few, tokens / (4 * rows)));
    const int64_t per = (tokens + chunks - 1) / chunks;
    return imax(rows, (per + rows - 1) / rows * rows);
}

#define TRIVANCE_NORM_SHAPES(RUN, RUN_LONG)                                                   \
    constexpr int V = kVec<T>;                                                                \
    switch (shape) {                                                                          \
        case Shape::kTiny: RUN(1, 8, 1); break;                                               \
        case Shape::k8: RUN(V, 8, 1); break;                                                  \
        case Shape::k16: RUN(V, 16, 1); break;                                                \
        case Shape::k32: RUN(V, 32, 1); break;                                                \
        case Shape::k64: RUN(V, 64, 1); break;                                                \
        case Shape::k64x2: RUN(V, 64, 2); break;                                              \
        case Shape::k64x4: if constexpr (V == 4) { RUN(V, 64, 4); } break;                        \
        case Shape::k256x2: RUN(V, 256, 2); break;                                            \
        case Shape::k256x4: if constexpr (V == 4) { RUN(V, 256, 4); } break;                      \
        case Shape::k512x2: if constexpr (V == 8) { RUN(V, 512, 2); } break;                      \
        case Shape::k512x4: RUN(V, 512, 4); break;                                            \
        case Shape::k512x8: if constexpr (V == 4) { RUN(V, 512, 8); } break;                      \
        case Shape::kLong: RUN_LONG(); break;                                                 \
    }

inline Shape shape_of(int64_t width, int dtype) {
    return dtype == TRIVANCE_F32 ? shape_of<float>(width) : shape_of<bf16>(width);
}

// Sizes that every call checks. The product of ranks, tokens and width stays within 2^60.
inline bool sizes_ok(int64_t ranks, int64_t tokens, int64_t width) {
    if (ranks < 1 || tokens < 0 || width < 1 || width > ((int64_t)1 << 24)) return false;
    return (__int128)ranks * (tokens + 1) * width < ((__int128)1 << 60);
}

// The chunks' sums, parts [ranks][chunks][sums][width], joined in the chunks' order, in 64 bits: the first into rows
// of dgamma, the second, if any, into rows of dbeta, both grad_rank apart (layernorm.hip).
int join_chunks(const float* parts, float* dgamma, float* dbeta, int sums, int64_t ranks, int64_t chunks,
                int64_t width, int64_t grad_rank, hipStream_t stream);

}  // namespace trivance
