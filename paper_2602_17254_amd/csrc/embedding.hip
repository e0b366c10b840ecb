// An embedding: rows of a table that all ranks hold, and each rank's gradient of that table.
//
//   y_t = scale table_{id_t}          dtable_v = scale sum of dy_t over the rank's tokens with id_t = v
//
// Memory bounds both: the gradient is dense, a row of the vector that an AllReduce sums, so most of its bytes are
// zeros. A few tokens are compared with each other. More are sorted by number (sort.hip, in one pass or two), and the
// launches of the sort, which latency bounds, write the zeros on the way. A number's tokens are then a run of the sorted ones.
// Groups of lanes take equal pieces of these, add up rows in the order of the tokens and write a row of the gradient where its
// run ends: no atomics, the same bits in every call. Sums of runs that go beyond a piece are joined in order in 64 bits.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "operators.h"
#include "sort.h"
#include "strips.h"
#include "vectors.h"

#pragma clang fp contract(fast)

namespace trivance {
namespace {

constexpr int64_t kMaxVocab = (int64_t)1 << 24;
constexpr int kThreads = 256;

struct Lookup {
    const void *ids, *table;
    int64_t ranks, tokens, vocab, width, table_row, y_rank, y_token;
    int wide, table_type;
    float scale;
    Share share;
};

__device__ __forceinline__ int64_t id_at(const void* ids, int wide, int64_t at) {
    return wide ? static_cast<const int64_t*>(ids)[at] : static_cast<const int*>(ids)[at];
}

constexpr int kLookupItems = 2;  // vectors of a lane: their numbers, then the table's rows, are on their way at once

// 38 us for 8 x 4096 tokens of 2048 bf16 from 32 bits, 134 MB written and 68 to 280 read, as rows repeat.
template <typename T, int V, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void lookup_kernel(Lookup a, T* y) {
    constexpr int U = kLookupItems;
    for_vectors<V, U>(a.share, a.ranks, a.tokens, a.width, [&](int64_t r, const Item(&item)[U]) {
        int64_t id[U];
        float v[U][V] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) id[u] = item[u].is ? id_at(a.ids, a.wide, r * a.tokens + item[u].token) : -1;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (id[u] >= 0 && id[u] < a.vocab)
                load_weights<V>(a.table, a.table_type, id[u] * a.table_row + item[u].first, INT64_MAX, 0.0f, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Some<T, V> o;
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = (T)(v[u][k] * a.scale);
            if (item[u].is) store_vector<STREAM, V>(y + r * a.y_rank + item[u].token * a.y_token + item[u].first, o);
        }
    });
}

template <typename T>
struct Table {
    const T* dy;
    float* dtable;  // a rank's rows follow one another
    const int *keys, *order;  // [ranks][tokens], sorted
    const int* counts;  // how many of a rank's tokens have a number, count_stride apart
    float* parts;  // [ranks][pieces][2][width]
    int64_t ranks, tokens, width, count_stride, dy_rank, dy_token, dtable_rank, pieces;
    int piece;
    float scale;
};

// A value of one of L lanes.
template <int L>
__device__ __forceinline__ int of_lane(int x, int lane) {
    if constexpr (L == 64) return __builtin_amdgcn_readlane(x, lane);
    return __shfl(x, lane, L);
}

// L lanes add up their columns of a piece of the sorted tokens, the next rows on their way meanwhile, and write a sum at the end of
// each run: to the gradient where the run lies in the piece, otherwise to the piece's parts, the first for a run that began
// before the piece, the second for one that ends behind it only. 50 us for 8 x 8192 tokens of 1024 bf16 (135 MB, and 113 written).
template <typename T, int L, bool STREAM>
__global__ __launch_bounds__(kThreads) void table_sums_kernel(Table<T> a) {
    constexpr int V = kVec<T>, G = kThreads / L, kAhead = 4;
    const int lane = threadIdx.x % L;
    const int64_t col = ((int64_t)blockIdx.x * L + lane) * V;
    int64_t piece = (int64_t)blockIdx.z * G + threadIdx.x / L;
    if constexpr (L == 64) piece = __builtin_amdgcn_readfirstlane((int)piece);  // the same in a wave
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* keys = a.keys + r * a.tokens;
        const int* order = a.order + r * a.tokens;
        const T* dy = a.dy + r * a.dy_rank;
        const int used = a.counts[r * a.count_stride];
        const int64_t first = piece * a.piece;
        if (first >= used) continue;
        const int end = (int)(first + a.piece < used ? first + a.piece : used);
        bool began = first == 0 || keys[first - 1] != keys[first];  // whether the run did in this piece
        float* part = a.parts + (r * a.pieces + piece) * 2 * a.width;
        float sum[V] = {};
        for_strips<L>((int)first, end, [&](int p0, int here) {
            const int own = p0 + (lane < here ? lane : 0);
            const int token = order[own], key = keys[own], after = own + 1 < used ? keys[own + 1] : -1;
            const auto fetch = [&](int p, typename Packed<T>::type(&v)[kAhead]) {
#pragma unroll
                for (int q = 0; q < kAhead; ++q)
                    if (p + q < here)
                        v[q] = load_columns<T, STREAM>(dy + of_lane<L>(token, p + q) * a.dy_token, col, a.width);
            };
            const auto add = [&](int p, const typename Packed<T>::type(&v)[kAhead]) {
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {
                    if (p + q >= here) break;
#pragma unroll
                    for (int k = 0; k < V; ++k) sum[k] += (float)v[q][k];
                    const int row = of_lane<L>(key, p + q);
                    const bool ends = of_lane<L>(after, p + q) != row;
                    if (!ends && p0 + p + q + 1 < end) continue;
                    float* to = part + (began ? a.width : 0);
                    if (began && ends) {
                        to = a.dtable + r * a.dtable_rank + row * a.width;
#pragma unroll
                        for (int k = 0; k < V; ++k) sum[k] *= a.scale;
                    }
                    store_row<float, V>(to, col, a.width, sum);
#pragma unroll
                    for (int k = 0; k < V; ++k) sum[k] = 0.0f;
                    began = true;
                }
            };
            typename Packed<T>::type even[kAhead], odd[kAhead];
            fetch(0, even);
            for (int p = 0; p < here; p += 2 * kAhead) {
                fetch(p + kAhead, odd);
                add(p, even);
                fetch(p + 2 * kAhead, even);
                add(p + kAhead, odd);
            }
        });
    }
}

// Few tokens need no sort. A wave takes a token and holds all numbers of its rank; where the token is the first with its number, it adds
// up the rows of all with that number, four at a time, joined in 64 bits, and writes the row, over the zeros that a launch
// before it wrote. 11 us for 9 x 128 tokens of 256 bf16 in place of 20 with a sort; 32 where all have the same number.
constexpr int kFewTokens = 128;

template <typename T>
__global__ __launch_bounds__(kThreads) void table_few_kernel(Table<T> a, const void* ids, int wide, int64_t vocab) {
    constexpr int V = kVec<T>, kStrips = kFewTokens / 64, kAhead = 4;
    const int lane = threadIdx.x % 64;
    const int t = __builtin_amdgcn_readfirstlane((int)(blockIdx.z * (kThreads / 64) + threadIdx.x / 64));
    if (t >= a.tokens) return;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        int key[kStrips];
#pragma unroll
        for (int s = 0; s < kStrips; ++s) {
            const int i = 64 * s + lane;
            const int64_t id = i < a.tokens ? id_at(ids, wide, r * a.tokens + i) : -1;
            key[s] = id >= 0 && id < vocab ? (int)id : -1;
        }
        int own = -1;
#pragma unroll
        for (int s = 0; s < kStrips; ++s)
            if (s == t / 64) own = __builtin_amdgcn_readlane(key[s], t % 64);
        if (own < 0) continue;
        uint64_t same[kStrips], before = 0;
#pragma unroll
        for (int s = 0; s < kStrips; ++s) {
            same[s] = __ballot(key[s] == own);
            if (s < t / 64) before |= same[s];
            else if (s == t / 64) before |= same[s] & ((1ull << t % 64) - 1);
        }
        if (before) continue;
        const T* dy = a.dy + r * a.dy_rank;
        double total[V] = {};
#pragma unroll
        for (int s = 0; s < kStrips; ++s) {
            const auto load = [&](uint64_t of) {
                const int64_t token = 64 * s + __ffsll((unsigned long long)of) - 1;
                return load_columns<T, false>(dy + token * a.dy_token, col, a.width);
            };
            uint64_t left = same[s];
            if (left && !(left & (left - 1))) {  // one, as mostly
                const auto v = load(left);
#pragma unroll
                for (int k = 0; k < V; ++k) total[k] += (float)v[k];
                continue;
            }
            while (left) {
                typename Packed<T>::type v[kAhead];
                float sum[V] = {};
                uint64_t next = left;
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {  // without a branch: the last row again where there are no more
                    v[q] = load(next);
                    next = next & (next - 1) ? next & (next - 1) : next;
                }
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {
                    const bool is = left != 0;
                    left &= left - 1;
#pragma unroll
                    for (int k = 0; k < V; ++k) sum[k] += is ? (float)v[q][k] : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < V; ++k) total[k] += sum[k];
            }
        }
        float out[V];
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = (float)total[k] * a.scale;
        store_row<float, V>(a.dtable + r * a.dtable_rank + own * a.width, col, a.width, out);
    }
}

// Blocks of zeros: a store a lane, as it has the highest rate; past the caches where the table is larger than they are.
constexpr int64_t kMaxZeros = (int64_t)1 << 21;

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void table_zeros_kernel(float* dtable, int64_t ranks, int64_t values, int64_t rank_stride) {
    const float zero[4] = {};
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y)
        for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4; i < values; i += (int64_t)gridDim.x * kThreads * 4)
            store_row<float, 4, STREAM>(dtable + r * rank_stride, i, values, zero);
}

constexpr int kJoinWaves = 4;
constexpr int kJoinPieces = 8;

// The rows of the runs that begin in a workgroup's pieces and end behind them: one at most in each. A wave adds up every
// fourth part of a run, eight loads on their way. Latency bounds it: 15 us for 8 x 256 pieces of 1024 columns.
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void table_join_kernel(Table<T> a) {
    __shared__ double sums[kJoinWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* keys = a.keys + r * a.tokens;
        const int used = a.counts[r * a.count_stride];
        for (int64_t piece0 = blockIdx.z * kJoinPieces; piece0 * a.piece < used; piece0 += gridDim.z * kJoinPieces) {
            // a lane looks at a piece that others follow; every wave does the same
            const int64_t first = (piece0 + lane) * a.piece, next = first + a.piece;
            int key = 0;
            bool begins = false;
            if (lane < kJoinPieces && next < used) {
                key = keys[next - 1];
                begins = keys[next] == key && (first == 0 || keys[first - 1] != key);
            }
            for (uint64_t found = __ballot(begins); found; found &= found - 1) {
                const int which = __ffsll((unsigned long long)found) - 1, row = __shfl(key, which, 64);
                const int64_t piece = piece0 + which;
                // the pieces that begin with the same number
                int64_t end = piece + 1;
                for (uint64_t all = ~0ull; all == ~0ull; ) {
                    const int64_t at = (end + lane) * a.piece;
                    all = __ballot(at < used && keys[at] == row);
                    end += all == ~0ull ? 64 : __ffsll((unsigned long long)~all) - 1;
                }
                double s = 0.0;
                if (col < a.width) {
                    const float* part = a.parts + r * a.pieces * 2 * a.width + col;
                    if (wave == 0) s = part[(2 * piece + 1) * a.width];
#pragma unroll 8
                    for (int64_t q = piece + 1 + wave; q < end; q += kJoinWaves) s += part[2 * q * a.width];
                }
                sums[wave][lane] = s;
                __syncthreads();
                if (wave == 0 && col < a.width) {
#pragma unroll
                    for (int w = 1; w < kJoinWaves; ++w) s += sums[w][lane];
                    a.dtable[r * a.dtable_rank + row * a.width + col] = (float)s * a.scale;
                }
                __syncthreads();
            }
        }
    }
}

int64_t imin(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t imax(int64_t a, int64_t b) { return a > b ? a : b; }

// Tokens of a piece: a power of two, from 32 on near an eighth of the root of the tokens' number, so that neither a piece's
// tokens nor a run's pieces are many: at most 2^17, of which a workgroup takes four or more. Pieces of 16 tokens took
// 239 us in place of 227 for 8 x 8192 tokens of 32000 numbers and 1024 columns, as more runs go beyond them.
int piece_of(int64_t tokens) {
    int64_t p = 32;
    while (64 * p * p < tokens || p << 17 < tokens) p *= 2;
    return (int)p;
}

int64_t pieces_of(int64_t tokens) { return (tokens + piece_of(tokens) - 1) / piece_of(tokens); }

// How the numbers are sorted: by their lower bits first, in a pass of its own, beyond kOnePass of them, unless a workgroup sorts all
// tokens of a rank. A pass's counters of many digits and chunks take longer to add up than two passes of fewer digits.
constexpr int64_t kOnePass = 1024;

struct Digits {
    int bits, bins, more;  // of the first pass (0: all); its digits; those of the second
};

Digits digits_of(int64_t ranks, int64_t tokens, int64_t vocab) {
    if (vocab <= kOnePass || (vocab <= kMaxBins && sort_launches(ranks, tokens, (int)vocab) == 1)) return {0, (int)vocab, 0};
    int bits = 0;
    while (((int64_t)1 << bits) < vocab) ++bits;
    bits = (bits + 1) / 2;
    return {bits, 1 << bits, (int)((vocab - 1) >> bits) + 1};
}

// What the workspace holds, in words of 4 bytes.
struct Places {
    int64_t offsets, keys[2], order[2], hist, parts, end;
};

Places places(int64_t ranks, int64_t tokens, int64_t width, int64_t vocab) {
    const Digits d = digits_of(ranks, tokens, vocab);
    Places p;
    int64_t at = 0;
    const auto take = [&](int64_t words) {
        const int64_t from = at;
        at += (words + 3) / 4 * 4;
        return from;
    };
    p.offsets = take(ranks * (d.bins + 1));
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = i == 0 || d.bits ? take(ranks * tokens) : p.keys[0];
        p.order[i] = i == 0 || d.bits ? take(ranks * tokens) : p.order[0];
    }
    p.hist = take(imax(sort_hist_values(ranks, tokens, d.bins), d.bits ? sort_hist_values(ranks, tokens, d.more) : 0));
    p.parts = take(tokens > kFewTokens ? ranks * pieces_of(tokens) * 2 * width : 0);  // few tokens have no pieces
    p.end = at;
    return p;
}

template <typename T>
int run_few(const Table<T>& a, const void* ids, int wide, int64_t vocab, hipStream_t stream) {
    const unsigned grid_y = (unsigned)imin(a.ranks, kShareMaxY);
    const int64_t values = vocab * a.width, blocks = imin((values + 4 * kThreads - 1) / (4 * kThreads), kMaxZeros);
    const dim3 zeros((unsigned)blocks, grid_y);
    if ((double)a.ranks * values * sizeof(float) > kStreamBytes)
        table_zeros_kernel<true><<<zeros, kThreads, 0, stream>>>(a.dtable, a.ranks, values, a.dtable_rank);
    else
        table_zeros_kernel<false><<<zeros, kThreads, 0, stream>>>(a.dtable, a.ranks, values, a.dtable_rank);
    const int rc = launch_status();
    if (rc || a.tokens == 0) return rc;
    constexpr int kWaves = kThreads / 64;
    const int64_t step = 64 * kVec<T>;
    const dim3 grid((unsigned)((a.width + step - 1) / step), grid_y, (unsigned)((a.tokens + kWaves - 1) / kWaves));
    table_few_kernel<T><<<grid, kThreads, 0, stream>>>(a, ids, wide, vocab);
    return launch_status();
}

bool sizes_ok(int64_t ranks, int64_t tokens, int64_t width, int64_t vocab) {
    if (ranks < 1 || tokens < 0 || width < 1 || width > ((int64_t)1 << 24) || vocab < 1) return false;
    return ranks <= INT32_MAX && (__int128)ranks * tokens <= INT32_MAX && (__int128)ranks * vocab * width < ((__int128)1 << 58);
}

template <typename T, typename F>
void with_lanes(int64_t width, F run) {
    const int64_t n = (width + kVec<T> - 1) / kVec<T>;
    if (n <= 8) run(std::integral_constant<int, 8>{});
    else if (n <= 16) run(std::integral_constant<int, 16>{});
    else if (n <= 32) run(std::integral_constant<int, 32>{});
    else run(std::integral_constant<int, 64>{});
}

template <typename T>
int run_gradient(const Table<T>& a, hipStream_t stream) {
    const unsigned grid_y = (unsigned)imin(a.ranks, kShareMaxY);
    with_lanes<T>(a.width, [&](auto l) {
        const int64_t step = (int64_t)l() * kVec<T>, rows = kThreads / l();
        const dim3 grid((unsigned)((a.width + step - 1) / step), grid_y, (unsigned)((a.pieces + rows - 1) / rows));
        if (a.ranks * a.tokens * a.width * (int64_t)sizeof(T) > kStreamBytes)
            table_sums_kernel<T, l(), true><<<grid, kThreads, 0, stream>>>(a);
        else
            table_sums_kernel<T, l(), false><<<grid, kThreads, 0, stream>>>(a);
    });
    const int rc = launch_status();
    if (rc) return rc;
    const dim3 grid((unsigned)((a.width + 63) / 64), grid_y,
                    (unsigned)imin((a.pieces + kJoinPieces - 1) / kJoinPieces, kShareMaxY));
    table_join_kernel<T><<<grid, 64 * kJoinWaves, 0, stream>>>(a);
    return launch_status();
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" {

int trivance_embedding_forward(const void* ids, const void* table, void* y, int64_t ranks, int64_t tokens,
                               int64_t width, int64_t vocab, int64_t table_row_stride, int64_t y_rank_stride,
                               int64_t y_token_stride, double scale, int dtype, int table_dtype, int id_dtype,
                               void* stream) {
    if (!is_float_type(dtype) || !is_float_type(table_dtype) || (id_dtype != TRIVANCE_I32 && id_dtype != TRIVANCE_I64))
        return TRIVANCE_EINVAL;
    if (!sizes_ok(ranks, tokens, width, vocab) || !std::isfinite((float)scale)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!ids || !table || !y || y == table || !rows_fit(1, vocab, width, 0, table_row_stride) ||
        !rows_fit(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_distinct(ranks, tokens, width, y_rank_stride, y_token_stride))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        return with_vector<T>(width, [&](auto v) {
            const Lookup a{ids, table, ranks, tokens, vocab, width, table_row_stride, y_rank_stride, y_token_stride,
                           id_dtype == TRIVANCE_I64, table_dtype, (float)scale,
                           share_vectors(ranks, tokens, width, v(), kLookupItems, false)};
            if (ranks * tokens * width * (int64_t)sizeof(T) > kStreamBytes)
                lookup_kernel<T, v(), true><<<a.share.grid, kShareThreads, 0, s>>>(a, static_cast<T*>(y));
            else
                lookup_kernel<T, v(), false><<<a.share.grid, kShareThreads, 0, s>>>(a, static_cast<T*>(y));
            return launch_status();
        });
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

int64_t trivance_embedding_workspace_bytes(int64_t ranks, int64_t tokens, int64_t width, int64_t vocab) {
    if (!sizes_ok(ranks, tokens, width, vocab)) return TRIVANCE_EINVAL;
    if (vocab > kMaxVocab) return TRIVANCE_EUNSUPPORTED;
    return places(ranks, tokens, width, vocab).end * (int64_t)sizeof(int);
}

int trivance_embedding_backward(const void* dy, const void* ids, float* dtable, int64_t ranks, int64_t tokens,
                                int64_t width, int64_t vocab, int64_t dy_rank_stride, int64_t dy_token_stride,
                                int64_t dtable_rank_stride, double scale, int dtype, int id_dtype, void* workspace,
                                int64_t workspace_bytes, void* stream) {
    if (!is_float_type(dtype) || (id_dtype != TRIVANCE_I32 && id_dtype != TRIVANCE_I64)) return TRIVANCE_EINVAL;
    const int64_t need = trivance_embedding_workspace_bytes(ranks, tokens, width, vocab);
    if (need < 0) return (int)need;
    if (!std::isfinite((float)scale)) return TRIVANCE_EINVAL;  // of zeros it would make no zeros
    if (!dtable || !rows_fit(ranks, 1, vocab * width, dtable_rank_stride, 0) ||
        !rows_distinct(ranks, 1, vocab * width, dtable_rank_stride, 0))
        return TRIVANCE_EINVAL;
    if (tokens > 0 && (!dy || !ids || dtable == dy || !rows_fit(ranks, tokens, width, dy_rank_stride, dy_token_stride)))
        return TRIVANCE_EINVAL;
    if (workspace_bytes < need || !workspace) return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(int)) return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (tokens <= kFewTokens) {
        const auto run = [&](auto type) {
            using T = decltype(type);
            return run_few(Table<T>{static_cast<const T*>(dy), dtable, nullptr, nullptr, nullptr, nullptr, ranks, tokens, width, 0,
                                    dy_rank_stride, dy_token_stride, dtable_rank_stride, 0, 0, (float)scale},
                           ids, id_dtype == TRIVANCE_I64, vocab, s);
        };
        return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
    }
    const Places at = places(ranks, tokens, width, vocab);
    int* words = static_cast<int*>(workspace);
    const Digits d = digits_of(ranks, tokens, vocab);
    const int first = sort_launches(ranks, tokens, d.bins), launches = first + (d.bits ? sort_launches(ranks, tokens, d.more) : 0);
    SortPass pass{};
    pass.ids = ids;
    pass.wide = id_dtype == TRIVANCE_I64;
    pass.ranks = ranks;
    pass.slots = tokens;
    pass.bound = vocab;
    pass.digits = d.bits ? d.bins - 1 : -1;
    pass.bins = d.bins;
    pass.offsets = words + at.offsets;
    pass.to_keys = words + at.keys[0];
    pass.to_order = words + at.order[0];
    pass.hist = words + at.hist;
    pass.zeros.at = dtable;
    pass.zeros.values = vocab * width;
    pass.zeros.rank_stride = dtable_rank_stride;
    if (const int rc = run_sort_pass(pass, s, 0, launches)) return rc;
    const int* counts = pass.offsets + pass.bins;
    if (d.bits) {
        SortPass next = pass;
        next.ids = nullptr;
        next.keys = pass.to_keys;
        next.order = pass.to_order;
        next.counts = counts;
        next.count_stride = pass.bins + 1;
        next.shift = d.bits;
        next.digits = -1;
        next.bins = d.more;
        next.offsets = nullptr;
        next.to_keys = words + at.keys[1];
        next.to_order = words + at.order[1];
        if (const int rc = run_sort_pass(next, s, first, launches)) return rc;
    }
    const auto run = [&](auto type) {
        using T = decltype(type);
        return run_gradient(
            Table<T>{static_cast<const T*>(dy), dtable, words + at.keys[1], words + at.order[1], counts,
                     reinterpret_cast<float*>(words + at.parts), ranks, tokens, width, pass.bins + 1, dy_rank_stride,
                     dy_token_stride, dtable_rank_stride, pieces_of(tokens), piece_of(tokens), (float)scale},
            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

}  // extern "C"
