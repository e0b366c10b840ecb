// A pass of a stable sort by counting. A rank's slots are cut into chunks of consecutive ones, a chunk into its waves'
// parts. The place of a key is the number of keys with smaller digits, and of those with its own digit in
// earlier chunks, in earlier waves of its chunk, in earlier rounds of 64 of its wave, and on lower lanes: sums of whole
// numbers, the same in every call.
// Latency bounds it: two launches (one where a workgroup takes all of a rank's slots), each a few dependent loads.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device.h"
#include "operators.h"
#include "sort.h"

namespace trivance {
namespace {

constexpr int64_t kMaxGridY = 65535;
constexpr int kHistThreads = 256;

// The key of a rank's slot, -1 for none.
__device__ __forceinline__ int key_of(const SortPass& a, int64_t r, int64_t i, int64_t used) {
    if (!a.ids) return i < used ? a.keys[r * a.slots + i] : -1;
    const int64_t at = r * a.slots + i;
    const int64_t id = a.wide ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int*>(a.ids)[at];
    bool is = id >= 0 && id < a.bound;
    if (a.mask) is = is && a.mask[r * a.tokens + fdiv32((uint32_t)i, a.by_top_k)];
    return is ? (int)id : -1;
}

__device__ __forceinline__ int digit_of(const SortPass& a, int key) { return (key >> a.shift) & a.digits; }

__device__ __forceinline__ int64_t used_of(const SortPass& a, int64_t r) {
    return a.ids ? a.slots : a.counts[r * a.count_stride];
}

__global__ __launch_bounds__(kHistThreads) void sort_count_kernel(SortPass a, int64_t per) {
    extern __shared__ int hist[];
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        for (int e = threadIdx.x; e < a.bins; e += kHistThreads) hist[e] = 0;
        __syncthreads();
        const int64_t begin = blockIdx.x * per, end = begin + per < a.slots ? begin + per : a.slots, used = used_of(a, r);
        for (int64_t i = begin + threadIdx.x; i < end; i += kHistThreads) {
            const int key = key_of(a, r, i, used);
            if (key >= 0) atomicAdd(&hist[digit_of(a, key)], 1);
        }
        __syncthreads();
        int* to = a.hist + (r * gridDim.x + blockIdx.x) * a.bins;
        for (int e = threadIdx.x; e < a.bins; e += kHistThreads) to[e] = hist[e];
        __syncthreads();
    }
}

// Local memory of a workgroup: a counter of each digit for each wave, the digits' first places, a value a wave.
__host__ __device__ constexpr int64_t place_words(int waves, int bins) { return (int64_t)(waves + 1) * bins + waves; }

__device__ __forceinline__ int wave_inclusive(int x) {
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d, 64);
        if ((int)(threadIdx.x % 64) >= d) x += y;
    }
    return x;
}

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void sort_place_kernel(SortPass a, int64_t per, int bits) {
    constexpr int kThreads = 64 * WAVES;
    extern __shared__ int shared[];
    int* first = shared;  // of each digit
    int* sums = shared + a.bins;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int* own = sums + WAVES + wave * a.bins;  // this wave's counters
    const int64_t chunks = gridDim.x, c = blockIdx.x;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t begin = c * per, end = begin + per < a.slots ? begin + per : a.slots, used = used_of(a, r);
        const int64_t from = begin + wave * (per / WAVES);
        const int64_t to = from + per / WAVES < end ? from + per / WAVES : end;
        for (int e = lane; e < a.bins; e += 64) own[e] = 0;
        __syncthreads();
        for (int64_t i = from + lane; i < to; i += 64) {
            const int key = key_of(a, r, i, used);
            if (key >= 0) atomicAdd(&own[digit_of(a, key)], 1);
        }
        __syncthreads();
        // each digit's keys before this chunk, and in all chunks; a wave's counter becomes the number before the wave
        for (int e = threadIdx.x; e < a.bins; e += kThreads) {
            int before = 0, all = 0;
            if (chunks > 1) {
                const int* h = a.hist + r * chunks * a.bins + e;
#pragma unroll 8
                for (int64_t k = 0; k < chunks; ++k) {
                    const int n = h[k * a.bins];
                    all += n;
                    before += k < c ? n : 0;
                }
            }
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                int* counter = sums + WAVES + w * a.bins + e;
                const int n = *counter;
                *counter = before;
                before += n;
            }
            first[e] = chunks > 1 ? all : before;
        }
        __syncthreads();
        // the digits' first places: a thread adds up consecutive digits, waves and workgroup the threads' sums
        const int each = (a.bins + kThreads - 1) / kThreads;
        const int e1 = threadIdx.x * each < (unsigned)a.bins ? threadIdx.x * each : a.bins;
        const int e2 = e1 + each < a.bins ? e1 + each : a.bins;
        int sum = 0;
        for (int e = e1; e < e2; ++e) sum += first[e];
        const int upto = wave_inclusive(sum);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int place = upto - sum, total = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) place += sums[w];
            total += sums[w];
        }
        for (int e = e1; e < e2; ++e) {
            const int n = first[e];
            first[e] = place;
            if (a.offsets && c == 0) a.offsets[r * (a.bins + 1) + e] = place;
            place += n;
        }
        if (a.offsets && c == 0 && threadIdx.x == 0) a.offsets[r * (a.bins + 1) + a.bins] = total;
        __syncthreads();
        constexpr int kAhead = 4;  // rounds of a wave whose keys are on their way at once
        for (int64_t base = from; base < to; base += 64 * kAhead) {
            int key[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t i = base + 64 * q + lane;
                key[q] = i < to ? key_of(a, r, i, used) : -1;
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t i = base + 64 * q + lane;
                const bool is = key[q] >= 0;
                const int d = is ? digit_of(a, key[q]) : 0;
                // the lanes with this lane's digit
                uint64_t same = __ballot(is);
                for (int b = 0; b < bits; ++b) {
                    const uint64_t set = __ballot(is && (d >> b & 1));
                    same &= d >> b & 1 ? set : ~set;
                }
                const int rank = (int)__popcll(same & ((1ull << lane) - 1));
                int at = -1;
                if (is) {
                    // all lanes read the counter before the last of them moves it on: a wave's accesses to local
                    // memory keep their order
                    const int n = __hip_atomic_load(&own[d], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    at = first[d] + n + rank;
                    if (rank + 1 == (int)__popcll(same))
                        __hip_atomic_store(&own[d], n + rank + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                }
                if (i < to) {
                    if (a.places) a.places[r * a.slots + i] = at;
                    if (a.to_order) {
                        if (is) a.to_order[r * a.slots + at] = a.ids ? (int)i : a.order[r * a.slots + i];
                        if (i >= total) a.to_order[r * a.slots + i] = -1;
                    }
                    if (a.to_keys && is) a.to_keys[r * a.slots + at] = key[q];
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace

// One workgroup for a rank's slots where its waves take at most eight rounds; otherwise chunks to fill the GPU, of one round of
// each wave at least, and no more than it takes little time to add up the counters of.
SortShape sort_shape(int64_t ranks, int64_t slots, int bins) {
    const auto rounded = [](int64_t n, int64_t to) { return (n + to - 1) / to * to; };
    int waves = bins <= 512 ? 16 : bins <= 2048 ? 4 : 2;
    if (slots <= waves * 64 * 8) return {waves, 1, rounded(slots > 0 ? slots : 1, waves * 64)};
    waves = bins <= 2048 ? 4 : 2;
    int64_t chunks = 1024 / ranks < 16 ? 16 : 1024 / ranks > 256 ? 256 : 1024 / ranks;
    if (chunks * bins > 65536) chunks = 65536 / bins;
    const int64_t per = rounded((slots + chunks - 1) / chunks, waves * 64);
    return {waves, (slots + per - 1) / per, per};
}

int64_t sort_hist_values(int64_t ranks, int64_t slots, int bins) {
    const int64_t chunks = sort_shape(ranks, slots, bins).chunks;
    return chunks > 1 ? ranks * chunks * bins : 0;
}

int run_sort_pass(const SortPass& a, hipStream_t stream) {
    const SortShape s = sort_shape(a.ranks, a.slots, a.bins);
    const dim3 grid((unsigned)s.chunks, (unsigned)(a.ranks < kMaxGridY ? a.ranks : kMaxGridY));
    int bits = 0;
    while ((1 << bits) < a.bins) ++bits;
    if (s.chunks > 1) {
        sort_count_kernel<<<grid, kHistThreads, sizeof(int) * a.bins, stream>>>(a, s.per);
        if (const int rc = launch_status()) return rc;
    }
    const size_t local = sizeof(int) * place_words(s.waves, a.bins);
    if (s.waves == 16) sort_place_kernel<16><<<grid, 64 * 16, local, stream>>>(a, s.per, bits);
    else if (s.waves == 4) sort_place_kernel<4><<<grid, 64 * 4, local, stream>>>(a, s.per, bits);
    else sort_place_kernel<2><<<grid, 64 * 2, local, stream>>>(a, s.per, bits);
    return launch_status();
}

}  // namespace trivance
