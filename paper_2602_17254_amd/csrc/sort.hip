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
constexpr int64_t kMaxZeros = (int64_t)1 << 21;  // workgroups of a launch that write zeros

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

// A workgroup's block of zeros, one of `most` of them, for every rank of its grid row; and the blocks that lie so many further on.
template <int THREADS>
__device__ __forceinline__ void fill_blocks(const SortPass& a, int64_t block, int64_t most) {
    const float zero[4] = {};
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y)
        for (int64_t b = block; b < a.zeros.blocks; b += most) {
            const int64_t begin = (a.zeros.first + b) * kZerosBlock;
            const int64_t end = begin + kZerosBlock < a.zeros.values ? begin + kZerosBlock : a.zeros.values;
            for (int64_t i = begin + threadIdx.x * 4; i < end; i += THREADS * 4)
                store_row<float, 4, true>(a.zeros.at + r * a.zeros.rank_stride, i, end, zero);
        }
}

__global__ __launch_bounds__(kHistThreads) void sort_count_kernel(SortPass a, int64_t per, int64_t chunks) {
    extern __shared__ int hist[];
    if (blockIdx.x >= chunks) return fill_blocks<kHistThreads>(a, blockIdx.x - chunks, gridDim.x - chunks);
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        for (int e = threadIdx.x; e < a.bins; e += kHistThreads) hist[e] = 0;
        __syncthreads();
        const int64_t begin = blockIdx.x * per, end = begin + per < a.slots ? begin + per : a.slots, used = used_of(a, r);
        for (int64_t i = begin + threadIdx.x; i < end; i += kHistThreads) {
            const int key = key_of(a, r, i, used);
            if (key >= 0) atomicAdd(&hist[digit_of(a, key)], 1);
        }
        __syncthreads();
        int* to = a.hist + (r * chunks + blockIdx.x) * a.bins;
        for (int e = threadIdx.x; e < a.bins; e += kHistThreads) to[e] = hist[e];
        __syncthreads();
    }
}

// Local memory of a workgroup: the digits' first places, a value a wave, a counter of each digit for each wave. A thread adds up
// consecutive first places: one word in 32 is left out, so that threads with 32 each do not meet in one bank.
__host__ __device__ constexpr int spread(int e) { return e + e / 32; }
__host__ __device__ constexpr int64_t place_words(int waves, int bins) { return spread(bins) + 1 + waves + (int64_t)waves * bins; }

__device__ __forceinline__ int wave_inclusive(int x) {
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d, 64);
        if ((int)(threadIdx.x % 64) >= d) x += y;
    }
    return x;
}

constexpr int kRounds = 2;  // of 64 slots, whose keys a wave holds in registers

// D: digits of a thread whose counters it adds up at once; more than one costs registers, and with them the rate of the
// zeros that other workgroups of the launch write.
template <int WAVES, int D>
__global__ __launch_bounds__(64 * WAVES) void sort_place_kernel(SortPass a, int64_t per, int64_t chunks, int bits) {
    constexpr int kThreads = 64 * WAVES, kCounters = D == 1 ? 16 : 8;
    if (blockIdx.x >= chunks) return fill_blocks<kThreads>(a, blockIdx.x - chunks, gridDim.x - chunks);
    extern __shared__ int shared[];
    int* first = shared;  // of each digit
    int* sums = shared + spread(a.bins) + 1;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int* own = sums + WAVES + wave * a.bins;  // this wave's counters
    const int64_t c = blockIdx.x;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t begin = c * per, end = begin + per < a.slots ? begin + per : a.slots, used = used_of(a, r);
        const int64_t from = begin + wave * (per / WAVES);
        const int64_t to = from + per / WAVES < end ? from + per / WAVES : end;
        int key[kRounds];
        const auto fetch = [&](int64_t base) {
#pragma unroll
            for (int q = 0; q < kRounds; ++q) {
                const int64_t i = base + 64 * q + lane;
                key[q] = i < to ? key_of(a, r, i, used) : -1;
            }
        };
        fetch(from);
        for (int e = lane; e < a.bins; e += 64) own[e] = 0;
        __syncthreads();
        for (int64_t base = from; base < to; base += 64 * kRounds) {
            if (base > from) fetch(base);
#pragma unroll
            for (int q = 0; q < kRounds; ++q)
                if (key[q] >= 0) atomicAdd(&own[digit_of(a, key[q])], 1);
        }
        __syncthreads();
        // each digit's keys before this chunk, and in all chunks; a wave's counter becomes the number before the wave
        for (int e0 = threadIdx.x; e0 < a.bins; e0 += D * kThreads) {
            int before[D] = {}, all[D] = {};
            if (chunks > 1) {
                const int* h = a.hist + r * chunks * a.bins + e0;
#pragma unroll kCounters
                for (int64_t k = 0; k < chunks; ++k)
#pragma unroll
                    for (int q = 0; q < D; ++q) {
                        const int n = q == 0 || e0 + q * kThreads < a.bins ? h[k * a.bins + q * kThreads] : 0;
                        all[q] += n;
                        before[q] += k < c ? n : 0;
                    }
            }
#pragma unroll
            for (int q = 0; q < D; ++q) {
                const int e = e0 + q * kThreads;
                if (e >= a.bins) break;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    int* counter = sums + WAVES + w * a.bins + e;
                    const int n = *counter;
                    *counter = before[q];
                    before[q] += n;
                }
                first[spread(e)] = chunks > 1 ? all[q] : before[q];
            }
        }
        __syncthreads();
        // the digits' first places: a thread adds up consecutive digits, waves and workgroup the threads' sums
        const int each = (a.bins + kThreads - 1) / kThreads;
        const int e1 = threadIdx.x * each < (unsigned)a.bins ? threadIdx.x * each : a.bins;
        const int e2 = e1 + each < a.bins ? e1 + each : a.bins;
        int sum = 0;
        for (int e = e1; e < e2; ++e) sum += first[spread(e)];
        const int upto = wave_inclusive(sum);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int place = upto - sum, total = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) place += sums[w];
            total += sums[w];
        }
        for (int e = e1; e < e2; ++e) {
            const int n = first[spread(e)];
            first[spread(e)] = place;
            if (a.offsets && c == 0) a.offsets[r * (a.bins + 1) + e] = place;
            place += n;
        }
        if (a.offsets && c == 0 && threadIdx.x == 0) a.offsets[r * (a.bins + 1) + a.bins] = total;
        __syncthreads();
        for (int64_t base = from; base < to; base += 64 * kRounds) {
            if (to - from > 64 * kRounds) fetch(base);
            // of each round the lanes with a lane's digit; the rounds' chains of steps are independent
            uint64_t same[kRounds];
#pragma unroll
            for (int q = 0; q < kRounds; ++q) same[q] = __ballot(key[q] >= 0);
            for (int b = 0; b < bits; ++b) {
#pragma unroll
                for (int q = 0; q < kRounds; ++q) {
                    const bool one = digit_of(a, key[q]) >> b & 1;  // of no key any will do
                    const uint64_t set = __ballot(one);
                    same[q] &= one ? set : ~set;
                }
            }
#pragma unroll
            for (int q = 0; q < kRounds; ++q) {
                const int64_t i = base + 64 * q + lane;
                const bool is = key[q] >= 0;
                const int rank = (int)__popcll(same[q] & ((1ull << lane) - 1));
                int at = -1;
                if (is) {
                    // all lanes read the counter before the last of them moves it on: a wave's accesses to local
                    // memory keep their order
                    const int d = digit_of(a, key[q]);
                    const int n = __hip_atomic_load(&own[d], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    at = first[spread(d)] + n + rank;
                    if (rank + 1 == (int)__popcll(same[q]))
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

// Chunks of as many slots as a workgroup's waves hold keys of, one where that is all; at most 128 (256 where they would be of more than
// four times as many slots), as each workgroup adds up the counters of all of them, and fewer of many digits. Both launches take
// 10 us for 8 ranks of 32768 slots and 64 digits, 20 for 131072 and 256.
SortShape sort_shape(int64_t ranks, int64_t slots, int bins) {
    const int waves = bins <= 2048 ? 4 : 2;
    const int64_t unit = waves * 64, full = unit * kRounds, chunks = slots > full * 4 * 128 ? 256 : 128;
    const int64_t most = 65536 / bins < chunks ? 65536 / bins : chunks;
    int64_t per = full * ((slots + full * most - 1) / (full * most));
    if (slots <= full) per = (slots + unit - 1) / unit * unit;
    if (per == 0) per = unit;
    return {waves, slots > per ? (slots + per - 1) / per : 1, per};
}

int64_t sort_hist_values(int64_t ranks, int64_t slots, int bins) {
    const int64_t chunks = sort_shape(ranks, slots, bins).chunks;
    return chunks > 1 ? ranks * chunks * bins : 0;
}

int sort_launches(int64_t ranks, int64_t slots, int bins) { return sort_shape(ranks, slots, bins).chunks > 1 ? 2 : 1; }

int run_sort_pass(SortPass a, hipStream_t stream, int launch, int launches) {
    const SortShape s = sort_shape(a.ranks, a.slots, a.bins);
    // this launch's share of the blocks of zeros
    const int64_t blocks = launches ? (a.zeros.values + kZerosBlock - 1) / kZerosBlock : 0;
    const auto grid = [&]() {
        a.zeros.first = launches ? blocks * launch / launches : 0;
        a.zeros.blocks = launches ? blocks * (launch + 1) / launches - a.zeros.first : 0;
        ++launch;
        const int64_t most = a.zeros.blocks < kMaxZeros ? a.zeros.blocks : kMaxZeros;
        return dim3((unsigned)(s.chunks + most), (unsigned)(a.ranks < kMaxGridY ? a.ranks : kMaxGridY));
    };
    int bits = 0;
    while ((1 << bits) < a.bins) ++bits;
    if (s.chunks > 1) {
        const dim3 g = grid();
        sort_count_kernel<<<g, kHistThreads, sizeof(int) * a.bins, stream>>>(a, s.per, s.chunks);
        if (const int rc = launch_status()) return rc;
    }
    const size_t local = sizeof(int) * place_words(s.waves, a.bins);
    const dim3 g = grid();
    if (a.bins <= 512) sort_place_kernel<4, 1><<<g, 64 * 4, local, stream>>>(a, s.per, s.chunks, bits);
    else if (s.waves == 4) sort_place_kernel<4, 4><<<g, 64 * 4, local, stream>>>(a, s.per, s.chunks, bits);
    else sort_place_kernel<2, 4><<<g, 64 * 2, local, stream>>>(a, s.per, s.chunks, bits);
    return launch_status();
}

}  // namespace trivance
