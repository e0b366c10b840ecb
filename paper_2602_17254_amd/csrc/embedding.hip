// An embedding: rows of a table that all ranks hold, and each rank's gradient of that table.
//
//   y_t = scale table_{id_t}          dtable_v = scale sum of dy_t over the rank's tokens with id_t = v
//
// Memory bounds both: the gradient is dense, a row of the vector that an AllReduce sums, so most of its bytes are
// zeros. A rank's tokens are sorted by number (sort.hip, one pass for tables of up to 4096 rows, otherwise two); a row's tokens
// are then a run of the sorted ones, and a group of lanes adds them up in the order of the tokens and writes the row
// once: no atomics, the same bits in every call. Frequent numbers have long runs: those of more than `piece` tokens are summed
// by pieces of that many, each by its own lanes, into the workspace, and the pieces' sums joined in order in 64 bits.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "operators.h"
#include "sort.h"
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

template <typename T, int V, bool STREAM>
__global__ __launch_bounds__(kShareThreads) void lookup_kernel(Lookup a, T* y) {
    for_vectors<V>(a.share, a.ranks, a.tokens, a.width, [&](int64_t r, int64_t t, int64_t i) {
        const int64_t id = id_at(a.ids, a.wide, r * a.tokens + t);
        float v[V] = {};
        if (id >= 0 && id < a.vocab)
            load_weights<V>(a.table, a.table_type, id * a.table_row + i, INT64_MAX, 0.0f, v);
        Some<T, V> o;
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = (T)(v[k] * a.scale);
        store_vector<STREAM, V>(y + r * a.y_rank + t * a.y_token + i, o);
    });
}

template <typename T>
struct Table {
    const T* dy;
    float* dtable;  // a rank's rows follow one another
    const int *keys, *order;  // [ranks][tokens], sorted
    const int* starts;  // [ranks][vocab + 1]: where each number's run starts
    float* parts;  // [ranks][pieces][2][width]
    int64_t ranks, tokens, vocab, width, dy_rank, dy_token, dtable_rank, pieces;
    int piece;
    float scale;
};

// Where the run of each number starts among a rank's sorted keys: the number of keys below it.
__global__ __launch_bounds__(kThreads) void starts_kernel(const int* keys, const int* counts, int64_t count_stride,
                                                          int* starts, int64_t ranks, int64_t tokens, int64_t vocab) {
    const int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (v > vocab) return;
    for (int64_t r = blockIdx.y; r < ranks; r += gridDim.y) {
        const int* k = keys + r * tokens;
        int low = 0, high = counts[r * count_stride];
        while (low < high) {
            const int mid = low + (high - low) / 2;
            if (k[mid] < v) low = mid + 1;
            else high = mid;
        }
        starts[r * (vocab + 1) + v] = low;
    }
}

// The sum of a lane's vector of dy over sorted tokens from .. to, four loads on their way at once.
template <typename T>
__device__ __forceinline__ void sum_run(const Table<T>& a, int64_t r, int from, int to, int64_t col, float (&sum)[kVec<T>]) {
    constexpr int V = kVec<T>, kAhead = 4;
    const int* order = a.order + r * a.tokens;
    const T* dy = a.dy + r * a.dy_rank;
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] = 0.0f;
    for (int p = from; p < to; p += kAhead) {
        typename Packed<T>::type v[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int at = p + q < to ? p + q : to - 1;
            v[q] = load_packed<T>(dy + (int64_t)order[at] * a.dy_token, col, a.width, (T)0.0f);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += p + q < to ? (float)v[q][k] : 0.0f;
    }
}

// L lanes take a row of the gradient, in tiles of columns where there are few rows.
template <typename T, int L, bool STREAM>
__global__ __launch_bounds__(kThreads) void table_rows_kernel(Table<T> a, int64_t tile) {
    constexpr int V = kVec<T>, G = kThreads / L;
    const int lane = threadIdx.x % L;
    const int64_t v = (int64_t)blockIdx.x * G + threadIdx.x / L;
    if (v >= a.vocab) return;
    const int64_t begin = blockIdx.z * tile, end = begin + tile < a.width ? begin + tile : a.width;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* starts = a.starts + r * (a.vocab + 1) + v;
        const int from = starts[0], to = starts[1];
        float* row = a.dtable + r * a.dtable_rank + v * a.width;
        if (from == to) {
            const float zero[4] = {};
            for (int64_t i = begin + lane * 4; i < end; i += L * 4) store_row<float, 4, STREAM>(row, i, end, zero);
        } else if (to - from <= a.piece) {
            for (int64_t i = begin + lane * V; i < end; i += L * V) {
                float sum[V];
                sum_run(a, r, from, to, i, sum);
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] *= a.scale;
                store_row<float, V, STREAM>(row, i, a.width, sum);
            }
        }
    }
}

// A piece's part of the long run that holds its first token, and of the one that holds its last.
template <typename T>
__global__ __launch_bounds__(kThreads) void table_pieces_kernel(Table<T> a) {
    constexpr int V = kVec<T>;
    const int64_t col = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * V, piece = blockIdx.z;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* starts = a.starts + r * (a.vocab + 1);
        const int* keys = a.keys + r * a.tokens;
        const int used = starts[a.vocab];
        const int64_t first = piece * a.piece;
        if (first >= used) continue;
        const int last = (int)(first + a.piece < used ? first + a.piece : used) - 1;
        const int k0 = keys[first], k1 = keys[last];
        float* part = a.parts + (r * a.pieces + piece) * 2 * a.width;
        float sum[V];
        if (starts[k0 + 1] - starts[k0] > a.piece) {
            const int to = starts[k0 + 1] <= last ? starts[k0 + 1] : last + 1;
            if (col < a.width) {
                sum_run(a, r, (int)first, to, col, sum);
                store_row<float, V>(part, col, a.width, sum);
            }
        }
        if (k1 != k0 && starts[k1 + 1] - starts[k1] > a.piece && col < a.width) {
            sum_run(a, r, starts[k1], last + 1, col, sum);
            store_row<float, V>(part + a.width, col, a.width, sum);
        }
    }
}

constexpr int kJoinWaves = 8;

// The row of the long run that starts in a piece, if one does: it holds the piece's last token. A wave adds up every eighth piece,
// eight loads on their way.
template <typename T>
__global__ __launch_bounds__(64 * kJoinWaves) void table_join_kernel(Table<T> a) {
    __shared__ double sums[kJoinWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane, piece = blockIdx.z;
    for (int64_t r = blockIdx.y; r < a.ranks; r += gridDim.y) {
        const int* starts = a.starts + r * (a.vocab + 1);
        const int used = starts[a.vocab];
        const int64_t first = piece * a.piece;
        if (first >= used) continue;
        const int last = (int)(first + a.piece < used ? first + a.piece : used) - 1;
        const int key = a.keys[r * a.tokens + last], from = starts[key], to = starts[key + 1];
        if (to - from <= a.piece || from < first) continue;
        const int64_t end = (to - 1) / a.piece;  // the run's last piece
        double s = 0.0;
        if (col < a.width) {
            const float* part = a.parts + r * a.pieces * 2 * a.width + col;
            // of its first piece the second sum, unless the piece starts with it
            if (wave == 0) s = part[(2 * piece + (from > first ? 1 : 0)) * a.width];
#pragma unroll 8
            for (int64_t q = piece + 1 + wave; q <= end; q += kJoinWaves) s += part[2 * q * a.width];
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && col < a.width) {
#pragma unroll
            for (int w = 1; w < kJoinWaves; ++w) s += sums[w][lane];
            a.dtable[r * a.dtable_rank + key * a.width + col] = (float)s * a.scale;
        }
        __syncthreads();
    }
}

int64_t imin(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t imax(int64_t a, int64_t b) { return a > b ? a : b; }

// Tokens of a piece: a power of two near the root of their number, so that neither a piece's tokens nor a run's pieces are
// many; at most 32768 pieces, the third dimension of a grid.
int piece_of(int64_t tokens) {
    int64_t p = 64;
    while (p * p < tokens) p *= 2;
    return (int)p;
}

// The bits of the numbers that the first of two passes sorts by; 0 for one pass.
int first_bits(int64_t vocab) {
    if (vocab <= kMaxBins) return 0;
    int bits = 0;
    while (((int64_t)1 << bits) < vocab) ++bits;
    return (bits + 1) / 2;
}

// What the workspace holds, in words of 4 bytes.
struct Places {
    int64_t starts, keys[2], order[2], offsets, hist, parts, end;
};

Places places(int64_t ranks, int64_t tokens, int64_t width, int64_t vocab) {
    const int bits = first_bits(vocab), passes = bits ? 2 : 1;
    const int bins = bits ? 1 << bits : (int)vocab, more = bits ? (int)((vocab - 1) >> bits) + 1 : 0;
    Places p;
    int64_t at = 0;
    const auto take = [&](int64_t words) {
        const int64_t from = at;
        at += (words + 3) / 4 * 4;
        return from;
    };
    p.starts = take(ranks * (vocab + 1));
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = i < passes ? take(ranks * tokens) : p.keys[0];
        p.order[i] = i < passes ? take(ranks * tokens) : p.order[0];
    }
    p.offsets = bits ? take(ranks * (bins + 1)) : p.starts;
    p.hist = take(imax(sort_hist_values(ranks, tokens, bins), more ? sort_hist_values(ranks, tokens, more) : 0));
    const int piece = piece_of(tokens);
    p.parts = take(tokens > piece ? ranks * ((tokens + piece - 1) / piece) * 2 * width : 0);
    p.end = at;
    return p;
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
    const bool beyond = (double)a.ranks * a.vocab * a.width * sizeof(float) > kStreamBytes;
    with_lanes<T>(a.width, [&](auto l) {
        const int64_t blocks = (a.vocab + kThreads / l() - 1) / (kThreads / l());
        // of tables with few rows several workgroups share a row's columns
        const int64_t step = (int64_t)l() * kVec<T>, columns = (a.width + step - 1) / step;
        const int64_t tiles = imin(columns, imax(1, 2048 / (blocks * grid_y)));
        const int64_t tile = (columns + tiles - 1) / tiles * step;
        const dim3 grid((unsigned)blocks, grid_y, (unsigned)((a.width + tile - 1) / tile));
        if (beyond) table_rows_kernel<T, l(), true><<<grid, kThreads, 0, stream>>>(a, tile);
        else table_rows_kernel<T, l(), false><<<grid, kThreads, 0, stream>>>(a, tile);
    });
    if (const int rc = launch_status()) return rc;
    if (a.tokens <= a.piece) return TRIVANCE_OK;  // no run is longer
    const int64_t step = (int64_t)kThreads * kVec<T>;
    table_pieces_kernel<T><<<dim3((unsigned)((a.width + step - 1) / step), grid_y, (unsigned)a.pieces), kThreads, 0, stream>>>(a);
    if (const int rc = launch_status()) return rc;
    table_join_kernel<T><<<dim3((unsigned)((a.width + 63) / 64), grid_y, (unsigned)a.pieces), 64 * kJoinWaves, 0, stream>>>(a);
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
    if (!sizes_ok(ranks, tokens, width, vocab)) return TRIVANCE_EINVAL;
    if (tokens == 0) return TRIVANCE_OK;
    if (!ids || !table || !y || !rows_fit(1, vocab, width, 0, table_row_stride) ||
        !rows_fit(ranks, tokens, width, y_rank_stride, y_token_stride) ||
        !rows_distinct(ranks, tokens, width, y_rank_stride, y_token_stride))
        return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto run = [&](auto type) {
        using T = decltype(type);
        return with_vector<T>(width, [&](auto v) {
            const Lookup a{ids, table, ranks, tokens, vocab, width, table_row_stride, y_rank_stride, y_token_stride,
                           id_dtype == TRIVANCE_I64, table_dtype, (float)scale, share_vectors(ranks, tokens, width, v())};
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
    if (!dtable || !rows_fit(ranks, 1, vocab * width, dtable_rank_stride, 0) ||
        !rows_distinct(ranks, 1, vocab * width, dtable_rank_stride, 0))
        return TRIVANCE_EINVAL;
    if (tokens > 0 && (!dy || !ids || !rows_fit(ranks, tokens, width, dy_rank_stride, dy_token_stride)))
        return TRIVANCE_EINVAL;
    if (workspace_bytes < need || !workspace) return TRIVANCE_ESIZE;
    if (reinterpret_cast<uintptr_t>(workspace) % sizeof(int)) return TRIVANCE_EINVAL;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Places at = places(ranks, tokens, width, vocab);
    int* words = static_cast<int*>(workspace);
    const int bits = first_bits(vocab);
    SortPass pass{};
    pass.ids = tokens > 0 ? ids : workspace;  // of no tokens nothing is read
    pass.wide = id_dtype == TRIVANCE_I64;
    pass.ranks = ranks;
    pass.slots = tokens;
    pass.bound = vocab;
    pass.digits = bits ? (1 << bits) - 1 : -1;
    pass.bins = bits ? 1 << bits : (int)vocab;
    pass.offsets = words + at.offsets;
    pass.to_keys = words + at.keys[0];
    pass.to_order = words + at.order[0];
    pass.hist = words + at.hist;
    if (const int rc = run_sort_pass(pass, s)) return rc;
    if (bits) {
        SortPass next = pass;
        next.ids = nullptr;
        next.keys = pass.to_keys;
        next.order = pass.to_order;
        next.counts = pass.offsets + pass.bins;
        next.count_stride = pass.bins + 1;
        next.shift = bits;
        next.digits = -1;
        next.bins = (int)((vocab - 1) >> bits) + 1;
        next.offsets = nullptr;
        next.to_keys = words + at.keys[1];
        next.to_order = words + at.order[1];
        if (const int rc = run_sort_pass(next, s)) return rc;
        starts_kernel<<<dim3((unsigned)((vocab + kThreads) / kThreads), (unsigned)imin(ranks, kShareMaxY)), kThreads, 0, s>>>(
            next.to_keys, next.counts, next.count_stride, words + at.starts, ranks, tokens, vocab);
        if (const int rc = launch_status()) return rc;
    }
    const auto run = [&](auto type) {
        using T = decltype(type);
        const int piece = piece_of(tokens);
        return run_gradient(
            Table<T>{static_cast<const T*>(dy), dtable, words + at.keys[bits ? 1 : 0], words + at.order[bits ? 1 : 0],
                     words + at.starts, reinterpret_cast<float*>(words + at.parts), ranks, tokens, vocab, width,
                     dy_rank_stride, dy_token_stride, dtable_rank_stride, (tokens + piece - 1) / piece, piece, (float)scale},
            s);
    };
    return dtype == TRIVANCE_F32 ? run(float{}) : dtype == TRIVANCE_BF16 ? run(bf16{}) : run(f16{});
}

}  // extern "C"
