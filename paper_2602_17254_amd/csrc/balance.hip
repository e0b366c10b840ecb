// The balance loss of a router with softmax probabilities, over the tokens of all ranks.
//
//   p_t = softmax(logits_t)     P_e = sum over tokens of p_te     c_e = slots that chose expert e
//   N = tokens that are not masked
//   loss = scale experts sum_e (c_e / (k N)) (P_e / N)
//   d loss / d logit_tj = p_tj (w_j - sum_e w_e p_te)     w_e = scale experts c_e / (k N^2)
//
// A rank counts its own tokens (counts and N in int32, P in fp32: rows that an AllReduce sums), and
// with the sums of all ranks forms the loss and its own tokens' gradient; counts have none.
// Memory bounds both passes over the logits. A token's logits lie in a group of 1 to 64 lanes, one or
// more 16-byte vectors each, so a row is read once and its maximum and sums are a few
// exchanges between lanes. A lane holds the same experts of every row: a workgroup's sums of
// probabilities add up in registers, its counts in local memory (integers: the order of
// additions does not matter); a second kernel joins the workgroups' sums in a fixed order, in 64 bits.
// Measured at 8 ranks of 32768 tokens: counts of 256 bf16 experts with two tokens in five unmasked, some 60 MB, 25
// us and 5 to join; gradient of 256 fp32 experts, 537 MB, 93 us (5.8 TB/s).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "device.h"
#include "operators.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = 4096;
constexpr int64_t kMaxGridX = 1 << 20;
constexpr int64_t kMaxGridY = 65535;

// exp(d) for d <= 0, to a few units in the last place at any distance from zero: two to the rounded product
// t = d log2(e), times exp of what the rounding left, d - t ln 2, which two terms of its series hold (ln 2's
// own rounding adds 5 units at the far end). NaN stays; below -104 the result is zero, and minus
// infinity would leave no number to correct with.
__device__ __forceinline__ float exp_below(float d) {
    constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
    d = __builtin_elementwise_maximum(d, -104.0f);
    const float t = d * kLog2E, p = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(p, __builtin_fmaf(-t, kLn2, d), p);
}

// A row's logits, as fp32, become exp(x - max); where every expert is excluded, by minus infinity, all are zero.
template <typename T, int L, int NV>
__device__ __forceinline__ void row_exp(float (&v)[NV][kVec<T>]) {
    constexpr int V = kVec<T>;
    float m = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) m = fmaxf(m, v[j][k]);
    m = lanes_max<L>(m);
    if (m == -__builtin_inff()) m = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) v[j][k] = exp_below(v[j][k] - m);
}

// One over a sum of exponentials; zero for the sum of none.
__device__ __forceinline__ float over(float s) { return s == 0.0f ? 0.0f : 1.0f / s; }

// A lane's part of every row: NV vectors, one every L vectors. What lies beyond the row's end is
// minus infinity: an excluded expert.
template <typename T, int L, int NV>
struct Row {
    typename Packed<T>::type v[NV];
    template <bool STREAM>
    __device__ __forceinline__ void fetch(const T* x, int lane, int experts) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            v[j] = load_packed<T, STREAM>(x, (j * L + lane) * kVec<T>, experts, (T)-__builtin_inff());
    }
    __device__ __forceinline__ void values(float (&out)[NV][kVec<T>]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < kVec<T>; ++k) out[j][k] = (float)v[j][k];
    }
};

template <typename T>
struct Counts {
    const T* logits;
    const void* ids;
    const uint8_t* mask;
    int* counts;   // rows `counts_rank` apart: the experts' counts, then the number of tokens
    float* probs;  // rows `probs_rank` apart
    int* part_counts;   // [ranks][chunks][experts + 1], where a rank's tokens are in several chunks
    float* part_probs;  // [ranks][chunks][experts]
    int64_t ranks, tokens, rank_stride, token_stride, counts_rank, probs_rank, chunks, per;  // per: most tokens of a chunk
    int experts, top_k, wide_ids;
    FastDiv32 by_top_k;
};

// A chunk's tokens are those of every `chunks`th group of rows, so that padding at the end of a rank's tokens
// leaves all workgroups the same work (28 us in place of 31 with contiguous chunks, at the size above). There the
// rows take half the time and what stands before and after them, with the join, the other half; more rows
// of a lane on their way at once were slower (30 us for two, 35 for four). With few tokens latency bounds it: 5.0 us
// at 9 ranks of 512 tokens and 64 experts.
template <typename T, int L, int NV>
__global__ __launch_bounds__(kThreads) void balance_counts_kernel(Counts<T> a) {
    constexpr int V = kVec<T>, G = kThreads / L;
    extern __shared__ int shared[];  // counts, then one float for each thread and value of a vector
    int* hist = shared;
    float* join = reinterpret_cast<float*>(shared + a.experts + 1);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int64_t c = blockIdx.x, step = a.chunks * G;
        const uint8_t* mask = a.mask ? a.mask + r * a.tokens : nullptr;
        __syncthreads();
        for (int e = threadIdx.x; e <= a.experts; e += kThreads) hist[e] = 0;
        __syncthreads();
        // the logits first, so that they are on their way during the counting
        Row<T, L, NV> next;
        const T* x = a.logits + r * a.rank_stride;
        int64_t t = c * G + group;
        const auto counted = [&](int64_t t) { return t < a.tokens && (!mask || mask[t]); };
        bool used = counted(t), after = counted(t + step);  // a token's mask is known before its row is fetched
        if (used) next.template fetch<false>(x + t * a.token_stride, lane, a.experts);
        const uint32_t most = (uint32_t)(a.per < a.tokens ? a.per : a.tokens);
        const uint32_t slots = most * (uint32_t)a.top_k;  // below 2^31, i0 below 2^32
        constexpr int kIds = 4;  // of a lane on their way at once
        for (uint32_t i0 = threadIdx.x; i0 < slots; i0 += kIds * kThreads) {
            int64_t id[kIds];
#pragma unroll
            for (int q = 0; q < kIds; ++q) {
                const uint32_t i = i0 + q * kThreads;
                id[q] = -1;
                if (i >= slots) continue;
                const uint32_t u = fdiv32(i, a.by_top_k);  // the slot's token among the chunk's
                const int64_t of = c * G + u / G * step + u % G;
                const int64_t at = (r * a.tokens + of) * a.top_k + (i - u * (uint32_t)a.top_k);
                if (counted(of))
                    id[q] = a.wide_ids ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int*>(a.ids)[at];
            }
#pragma unroll
            for (int q = 0; q < kIds; ++q)
                if (id[q] >= 0 && id[q] < a.experts) atomicAdd(&hist[id[q]], 1);
        }
        float sum[NV][V] = {};
        int live = 0;
        while (t < a.tokens) {
            const bool use = used;
            float v[NV][V];
            next.values(v);
            t += step;
            used = after;
            if (used) next.template fetch<false>(x + t * a.token_stride, lane, a.experts);
            after = counted(t + step);
            if (!use) continue;
            row_exp<T, L, NV>(v);
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) s += v[j][k];
            const float inv = over(lanes_sum<L>(s));
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) sum[j][k] += v[j][k] * inv;
            ++live;
        }
        if (lane == 0 && live) atomicAdd(&hist[a.experts], live);
        float* probs = a.chunks > 1 ? a.part_probs + (r * a.chunks + c) * a.experts
                                    : a.probs + r * a.probs_rank;
        int* counts = a.chunks > 1 ? a.part_counts + (r * a.chunks + c) * (a.experts + 1)
                                   : a.counts + r * a.counts_rank;
        // the groups' sums in the groups' order, up to 256 of them, in 64 bits; one vector of each lane at a time
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < V; ++k) join[group * L * V + lane * V + k] = sum[j][k];
            __syncthreads();
            for (int i = threadIdx.x; i < L * V; i += kThreads) {
                const int e = j * L * V + i;
                if (e >= a.experts) break;
                double s = 0.0;
                for (int g = 0; g < G; ++g) s += join[g * L * V + i];
                probs[e] = (float)s;
            }
        }
        for (int e = threadIdx.x; e <= a.experts; e += kThreads) counts[e] = hist[e];
    }
}

constexpr int kJoinWaves = 8;

// Columns 0 .. experts - 1 join the sums of probabilities, the next experts + 1 the counts. Eight waves share
// the chunks of 64 columns, eight loads of each on their way: latency bounds it (4.1 us for 8 ranks of 256 chunks).
__global__ __launch_bounds__(64 * kJoinWaves) void balance_join_kernel(
    const int* part_counts, const float* part_probs, int* counts, float* probs, int64_t ranks,
    int64_t chunks, int experts, int64_t counts_rank, int64_t probs_rank) {
    __shared__ double sums[kJoinWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int col = blockIdx.x * 64 + lane;
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y) {
        double s = 0.0;  // exact for the counts
        if (col < experts) {
            const float* p = part_probs + r * chunks * experts + col;
#pragma unroll 8
            for (int64_t c = wave; c < chunks; c += kJoinWaves) s += p[c * experts];
        } else if (col < 2 * experts + 1) {
            const int* p = part_counts + r * chunks * (experts + 1) + (col - experts);
#pragma unroll 8
            for (int64_t c = wave; c < chunks; c += kJoinWaves) s += p[c * (experts + 1)];
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && col < 2 * experts + 1) {
#pragma unroll
            for (int w = 1; w < kJoinWaves; ++w) s += sums[w][lane];
            if (col < experts) probs[r * probs_rank + col] = (float)s;
            else counts[r * counts_rank + (col - experts)] = (int)s;
        }
        __syncthreads();
    }
}

// scale experts / (k N^2), what a count is multiplied by; zero where no token is left.
__device__ __forceinline__ double count_weight(int tokens, int experts, int64_t top_k, double scale) {
    const double n = tokens;
    return tokens > 0 ? scale * experts / ((double)top_k * n * n) : 0.0;
}

// One workgroup a rank, an expert a lane. Latency bounds it: 2.6 us at 9 ranks of 64 experts.
__global__ __launch_bounds__(kThreads) void balance_loss_kernel(const int* counts, const float* probs,
                                                                float* loss, int64_t ranks, int experts,
                                                                int64_t top_k, int64_t counts_rank,
                                                                int64_t probs_rank, double scale) {
    __shared__ double sums[kThreads / 64];
    for (int64_t r = blockIdx.x; r < ranks; r += gridDim.x) {
        const int* c = counts + r * counts_rank;
        const float* p = probs + r * probs_rank;
        const int tokens = c[experts];
        double s = 0.0;
        for (int e = threadIdx.x; e < experts; e += kThreads) s += (double)c[e] * p[e];
        s = lanes_sum<64>(s);
        if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            loss[r] = tokens > 0 ? (float)(s * count_weight(tokens, experts, top_k, scale)) : 0.0f;
        }
        __syncthreads();
    }
}

template <typename T>
struct Gradient {
    const T* logits;
    const int* counts;
    const uint8_t* mask;
    const float* dloss;
    T* dlogits;
    int64_t ranks, tokens, rank_stride, token_stride, d_rank, d_token, counts_rank, top_k;
    double scale;
    int experts;
};

// Bound by the bytes of the logits and of their gradient. Both go past the caches where they would not
// stay in them (STREAM): 95 us against 100 at 8 x 32768 x 256 fp32. The counts read the logits once and
// lose by it, 37 us against 31 at the same size in bf16, so they never do.
template <typename T, int L, int NV, bool STREAM>
__global__ __launch_bounds__(kThreads) void balance_gradient_kernel(Gradient<T> a) {
    constexpr int V = kVec<T>, G = kThreads / L;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* counts = a.counts + r * a.counts_rank;
        const uint8_t* mask = a.mask ? a.mask + r * a.tokens : nullptr;
        const int64_t step = (int64_t)gridDim.x * G;
        Row<T, L, NV> next;
        const T* x = a.logits + r * a.rank_stride;
        int64_t t = (int64_t)blockIdx.x * G + group;
        const auto counted = [&](int64_t t) { return t < a.tokens && (!mask || mask[t]); };
        bool used = counted(t), after = counted(t + step);  // a token's mask is known before its row is fetched
        if (used) next.template fetch<STREAM>(x + t * a.token_stride, lane, a.experts);
        const float f = (float)(count_weight(counts[a.experts], a.experts, a.top_k, a.scale) *
                                (a.dloss ? (double)a.dloss[r] : 1.0));
        float w[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int e = (j * L + lane) * V + k;
                w[j][k] = e < a.experts ? f * (float)counts[e] : 0.0f;
            }
        while (t < a.tokens) {
            const bool use = used;
            T* d = a.dlogits + r * a.d_rank + t * a.d_token;
            float v[NV][V];
            next.values(v);
            t += step;
            used = after;
            if (used) next.template fetch<STREAM>(x + t * a.token_stride, lane, a.experts);
            after = counted(t + step);
            if (use) {
                row_exp<T, L, NV>(v);
                float s = 0.0f, q = 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        s += v[j][k];
                        q += v[j][k] * w[j][k];
                    }
                const float inv = over(lanes_sum<L>(s));
                q = lanes_sum<L>(q) * inv;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int k = 0; k < V; ++k) v[j][k] = v[j][k] * inv * (w[j][k] - q);
            } else {  // what lies there is not read
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int k = 0; k < V; ++k) v[j][k] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
                store_row<T, V, STREAM>(d, (int64_t)(j * L + lane) * V, a.experts, v[j]);
        }
    }
}

int64_t imin(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t imax(int64_t a, int64_t b) { return a > b ? a : b; }

// Lanes of a row: a power of two that holds its vectors, at most a wave.
int row_lanes(int experts, int vec) {
    const int n = (experts + vec - 1) / vec;
    int l = 1;
    while (l < n && l < 64) l *= 2;
    return l;
}

// The most tokens of a chunk: enough chunks to fill the GPU, but four rows at least for each group of lanes.
int64_t chunk_tokens(int64_t ranks, int64_t tokens, int lanes) {
    const int64_t rows = kThreads / lanes;
    const int64_t chunks = imax(1, imin((2048 + ranks - 1) / ranks, tokens / (4 * rows)));
    const int64_t per = (tokens + chunks - 1) / chunks;
    return imax(rows, (per + rows - 1) / rows * rows);
}

// Groups of 1 to 64 lanes with one vector each, then waves with more. A row of 4096 experts takes 16 of
// fp32 or 8 of 16 bits.
template <typename T, typename F>
void with_shape(int experts, F run) {
    constexpr int V = kVec<T>;
    const int n = (experts + V - 1) / V;
#define CASE(L, NV) return run(std::integral_constant<int, L>{}, std::integral_constant<int, NV>{})
    if (n <= 1) CASE(1, 1);
    if (n <= 2) CASE(2, 1);
    if (n <= 4) CASE(4, 1);
    if (n <= 8) CASE(8, 1);
    if (n <= 16) CASE(16, 1);
    if (n <= 32) CASE(32, 1);
    if (n <= 64) CASE(64, 1);
    if (n <= 128) CASE(64, 2);
    if (n <= 256) CASE(64, 4);
    if (n <= 512) CASE(64, 8);
    if constexpr (V == 4) CASE(64, 16);
#undef CASE
}

template <typename T>
int run_counts(const Counts<T>& a, hipStream_t stream) {
    const dim3 grid((unsigned)a.chunks, (unsigned)imin(a.ranks, kMaxGridY));
    const size_t local = sizeof(int) * (a.experts + 1 + kThreads * kVec<T>);
    with_shape<T>(a.experts, [&](auto l, auto nv) {
        balance_counts_kernel<T, l(), nv()><<<grid, kThreads, local, stream>>>(a);
    });
    const int rc = launch_status();
    if (rc || a.chunks == 1) return rc;
    const dim3 join((unsigned)((2 * a.experts + 1 + 63) / 64), (unsigned)imin(a.ranks, kMaxGridY));
    balance_join_kernel<<<join, 64 * kJoinWaves, 0, stream>>>(a.part_counts, a.part_probs, a.counts,
                                                              a.probs, a.ranks, a.chunks, a.experts,
                                                              a.counts_rank, a.probs_rank);
    return launch_status();
}

template <typename T>
int run_gradient(const Gradient<T>& a, hipStream_t stream) {
    const int rows = kThreads / row_lanes(a.experts, kVec<T>);
    // about 64 workgroups for each of the 256 compute units, with the same number of rows each
    const int64_t units = (a.tokens + rows - 1) / rows, most = imax(1, 256 * 64 / a.ranks);
    const int64_t each = (units + most - 1) / most;
    const dim3 grid((unsigned)((units + each - 1) / each), (unsigned)imin(a.ranks, kMaxGridY));
    with_shape<T>(a.experts, [&](auto l, auto nv) {
        if (a.ranks * a.tokens * a.experts * (int64_t)sizeof(T) > kStreamBytes)
            balance_gradient_kernel<T, l(), nv(), true><<<grid, kThreads, 0, stream>>>(a);
        else
            balance_gradient_kernel<T, l(), nv(), false><<<grid, kThreads, 0, stream>>>(a);
    });
    return launch_status();
}

// Sizes that every call checks: the numbers of tokens and of slots of all ranks fit an int32 count.
bool sizes_ok(int64_t ranks, int64_t tokens, int64_t experts, int64_t top_k) {
    if (ranks < 1 || tokens < 0 || experts < 1 || top_k < 1) return false;
    return (__int128)ranks * tokens * top_k <= INT32_MAX && ranks <= INT32_MAX && top_k <= INT32_MAX;
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" {

int64_t trivance_balance_workspace_bytes(int64_t ranks, int64_t tokens, int64_t experts) {
    if (!sizes_ok(ranks, tokens, experts, 1)) return TRIVANCE_EINVAL;
    if (experts > kMaxExperts) return TRIVANCE_EUNSUPPORTED;
    int64_t most = 0;
    for (const int vec : {kVec<float>, kVec<bf16>}) {
        const int64_t per = chunk_tokens(ranks, tokens, row_lanes((int)experts, vec));
        const int64_t chunks = imax(1, (tokens + per - 1) / per);
        if (chunks > 1) most = imax(most, ranks * chunks * (2 * experts + 1) * (int64_t)sizeof(int));
    }
    return most;
}

int trivance_balance_counts(const void* logits, const void* chosen, const uint8_t* mask,
                            int32_t* counts, float* probs, int64_t ranks, int64_t tokens,
                            int64_t experts, int64_t top_k, int64_t rank_stride,
                            int64_t token_stride, int64_t counts_rank_stride,
                            int64_t probs_rank_stride, int dtype, int id_dtype, void* workspace,
                            int64_t workspace_bytes, void* stream) {
    if (!is_float_type(dtype) || (id_dtype != TRIVANCE_I32 && id_dtype != TRIVANCE_I64))
        return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, experts, top_k)) return TRIVANCE_EINVAL;
    if (experts > kMaxExperts) return TRIVANCE_EUNSUPPORTED;
    if (!counts || !probs || !rows_fit(ranks, 1, experts + 1, counts_rank_stride, 0) ||
        !rows_distinct(ranks, 1, experts + 1, counts_rank_stride, 0) ||
        !rows_fit(ranks, 1, experts, probs_rank_stride, 0) ||
        !rows_distinct(ranks, 1, experts, probs_rank_stride, 0))
        return TRIVANCE_EINVAL;
    if (tokens > 0 && (!logits || !chosen ||
                       !rows_fit(ranks, tokens, experts, rank_stride, token_stride)))
        return TRIVANCE_EINVAL;
    const int64_t need = trivance_balance_workspace_bytes(ranks, tokens, experts);
    if (workspace_bytes < need || (need > 0 && !workspace)) return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(int)) return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        const int64_t per = chunk_tokens(ranks, tokens, row_lanes((int)experts, kVec<T>));
        const int64_t chunks = imax(1, (tokens + per - 1) / per);
        int* part = static_cast<int*>(workspace);
        return run_counts(
            Counts<T>{static_cast<const T*>(logits), chosen, mask, counts, probs, part,
                      reinterpret_cast<float*>(part + ranks * chunks * (experts + 1)), ranks, tokens,
                      rank_stride, token_stride, counts_rank_stride, probs_rank_stride, chunks, per,
                      (int)experts, (int)top_k, id_dtype == TRIVANCE_I64,
                      make_fastdiv32((uint32_t)top_k)},
            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

int trivance_balance_loss(const int32_t* counts, const float* probs, float* loss, int64_t ranks,
                          int64_t experts, int64_t top_k, int64_t counts_rank_stride,
                          int64_t probs_rank_stride, double scale, void* stream) {
    if (!sizes_ok(ranks, 0, experts, top_k)) return TRIVANCE_EINVAL;
    if (experts > kMaxExperts) return TRIVANCE_EUNSUPPORTED;
    if (!counts || !probs || !loss || !rows_fit(ranks, 1, experts + 1, counts_rank_stride, 0) ||
        !rows_fit(ranks, 1, experts, probs_rank_stride, 0))
        return TRIVANCE_EINVAL;
    balance_loss_kernel<<<(unsigned)imin(ranks, kMaxGridX), kThreads, 0, reinterpret_cast<hipStream_t>(stream)>>>(
        counts, probs, loss, ranks, (int)experts, top_k, counts_rank_stride, probs_rank_stride, scale);
    return launch_status();
}

int trivance_balance_backward(const void* logits, const int32_t* counts, const uint8_t* mask,
                              const float* dloss, void* dlogits, int64_t ranks, int64_t tokens,
                              int64_t experts, int64_t top_k, int64_t rank_stride,
                              int64_t token_stride, int64_t d_rank_stride, int64_t d_token_stride,
                              int64_t counts_rank_stride, double scale, int dtype, void* stream) {
    if (!is_float_type(dtype) || !sizes_ok(ranks, tokens, experts, top_k)) return TRIVANCE_EINVAL;
    if (experts > kMaxExperts) return TRIVANCE_EUNSUPPORTED;
    if (tokens == 0) return TRIVANCE_OK;
    if (!logits || !counts || !dlogits || !rows_fit(ranks, tokens, experts, rank_stride, token_stride) ||
        !rows_fit(ranks, 1, experts + 1, counts_rank_stride, 0) ||
        !rows_fit(ranks, tokens, experts, d_rank_stride, d_token_stride) ||
        !rows_distinct(ranks, tokens, experts, d_rank_stride, d_token_stride))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        return run_gradient(Gradient<T>{static_cast<const T*>(logits), counts, mask, dloss,
                                        static_cast<T*>(dlogits), ranks, tokens, rank_stride,
                                        token_stride, d_rank_stride, d_token_stride,
                                        counts_rank_stride, top_k, scale, (int)experts},
                            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

}  // extern "C"
