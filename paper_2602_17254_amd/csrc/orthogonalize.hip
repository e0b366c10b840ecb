// Orthogonalises matrices by Newton-Schulz products: X0 = G / (|G|_F + eps), and per step
//
//   A = X X'     P = b A + c A A     X <- a X + P X
//
// on the smaller side of G (X = G' where G is taller than wide), so that every singular value s of X0
// passes the odd polynomial a s + b s^3 + c s^5 of each step and the singular vectors stay.
//
// Precision. A weak direction of G grows by up to a in every step (by 485 in five steps with
// a = 3.4445), and so does any rounding noise that falls into it: with bf16 operands five steps end 1
// to 30% off, with fp16 0.1 to 3%, by the spectrum. Every matrix is kept as two fp16 numbers hi + lo of
// 22 bits together, and a product is three MFMA products hi hi + hi lo + lo hi in fp32 sums: fp32
// accuracy for every spectrum at a third of the fp16 rate, five times the rate of fp32 MFMA. Small
// entries, which lo holds with a fixed spacing, decide how near that comes: X, A and P are each held times
// the largest power of two that their range allows, 2^15, 2^15 and 2^13 for the usual coefficients. a X, the largest
// term of an early step, joins when the sum is done, which would round at its size in every addition
// (one step of 4000 x 4000 fp32: 5 times the error of fp32 products with a in P, 0.6 times without). Five steps
// are 0.5 to 0.8 times as far off as fp32 products from 512 rows on. X is
// formed in every step: a form that carried A <- A P P through three steps, at two thirds of the time,
// lost the singular values whose squares fall into A's rounding (2.2 times the error of fp32 products at
// 2048 x 8192). G enters scaled by a power
// of two, exactly where it has 16 bits; the rest of the norm goes into the first step's coefficients.
//
// What bounds it: the MFMA rate, for matrices of some hundred rows and more; below that the latency of the steps'
// launches one after another, or of one workgroup's. Five steps measured: 2048 x 8192 bf16 2.05 ms, 0.27 PFLOP/s
// of the products' own and 0.56 to 1.0 of MFMA in each kernel; 1024 x 4096 0.47 ms; 512 x 512 fp32 0.14;
// 64 x 2048 0.066; 64 x 256 0.041.
// Layout. X is kept both ways round, so that both operands of every product have their summed index
// contiguous; sides are padded with zeros to whole tiles. A and A A are symmetric: only tiles on and
// above the diagonal are computed and each is written to both places.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "device.h"
#include "operators.h"
#include "orthogonalize_plan.h"

namespace trivance {
namespace {

constexpr int kMaxSteps = 64;
constexpr int64_t kMaxSide = 1 << 16;
constexpr int kNormParts = 1024;  // most partial sums of a matrix's norm

typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef f16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

// A matrix in two planes, rows `ld` apart.
struct Planes {
    f16 *hi, *lo;
    int64_t batch;  // elements from one matrix to the next
    int ld;
};

// Of a step, times the scales of what they multiply and make: P as stored is
// b (A as stored) + c (the sums of products of A as stored), X as stored becomes a X + P X.
struct Coefficients {
    float a, b, c;
};

// Of one matrix: the first step's coefficients, and where its norm lies below eps, by which power of two X is
// held larger than it is: held as it is, it would sink into the fixed spacing of lo (1e-3 off for norms of
// 1e-14 and eps 1e-7).
struct Start {
    Coefficients k;
    int shift;
};

// A step of matrices held 2^shift too large at the start. What the steps before this one and it itself
// raise X by at most, 2^before and 2^after, is taken off until nothing is left, so that X stays near one.
__device__ __forceinline__ int shift_left(int shift, int grown) { return shift > grown ? shift - grown : 0; }

__device__ __forceinline__ Coefficients shifted(Coefficients k, int shift, int before, int after) {
    const int s = shift_left(shift, before), t = shift_left(shift, after);
    return {ldexpf(k.a, t - s), ldexpf(k.b, t - 3 * s), ldexpf(k.c, t - 5 * s)};
}

template <typename T>
struct Input {
    const T* x;
    int64_t batch;
    int64_t si, sj;  // strides of X's rows and columns
    int m, n;        // X is m x n, m <= n
};

__device__ __forceinline__ void split(float v, f16& hi, f16& lo) {
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

// Partial sums of squares in 64 bits, so that no finite matrix overflows. Rows of the input as it lies in
// memory, in pieces of 256 vectors. 11 us at 2048 x 8192 bf16, 34 MB, and 4 where latency bounds it.
template <typename T>
__global__ __launch_bounds__(256) void norm_parts_kernel(Input<T> in, double* parts) {
    constexpr int V = kVec<T>;
    __shared__ double sums[4];
    const bool tall = in.sj != 1;
    const int rows = tall ? in.n : in.m, cols = tall ? in.m : in.n;
    const int64_t stride = tall ? in.sj : in.si;
    const T* x = in.x + blockIdx.y * in.batch;
    const int pieces = (cols + 256 * V - 1) / (256 * V);
    double s = 0.0;
    for (int64_t u = blockIdx.x; u < (int64_t)rows * pieces; u += gridDim.x) {
        float v[V];
        load_row<T>(x + u / pieces * stride, (u % pieces * 256 + threadIdx.x) * V, cols, 0.0f, v);
#pragma unroll
        for (int k = 0; k < V; ++k) s += (double)v[k] * (double)v[k];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        parts[blockIdx.y * kNormParts + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The power of two 2^e above the norm, and the first step's coefficients, which hold what is left of it:
// zeros for a zero matrix, not a number where the norm is none. `grown`: of the first step.
__device__ __forceinline__ void scale_of(double squares, Coefficients c, double eps, int grown, int& e, Start& start) {
    const double norm = sqrt(squares);
    e = norm > 0.0 && norm < __builtin_inf() ? ilogb(norm) + 1 : 0;
    const double alpha = norm == 0.0 ? 0.0
                         : norm < __builtin_inf() ? ldexp(1.0, e) / (norm + eps)
                                                  : __builtin_nan("");
    start.shift = alpha > 0.0 && alpha < 0.5 ? -ilogb(alpha) - 1 : 0;
    const double first = ldexp(alpha, shift_left(start.shift, grown)), square = alpha * alpha;
    start.k = {(float)(c.a * first), (float)(c.b * first * square), (float)(c.c * first * square * square)};
}

// X both ways round, scaled by 2^scale over the power of two above the norm and padded with zeros, and the
// first step's coefficients. A workgroup takes 64 x 64 values, read as they lie in memory. 32 us at 2048 x 8192
// bf16, 34 MB read and 67 written (3 TB/s, 3% of the call): stores of 128 bytes a row bound it.
template <typename T>
__global__ __launch_bounds__(256) void split_kernel(Input<T> in, const double* parts, int nparts,
                                                    Planes x, Planes xt, int scale, Coefficients c, double eps,
                                                    int grown, Start* start) {
    constexpr int V = kVec<T>, kRow = 64 + 8;
    __shared__ half8 tiles[2][64 * kRow / 8];
    const int64_t b = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x % 64; i < nparts; i += 64) sum += parts[b * kNormParts + i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    int e;
    Start mine;
    scale_of(sum, c, eps, grown, e, mine);
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    if (i0 == 0 && j0 == 0 && threadIdx.x == 0) start[b] = mine;
    // rows and columns as in memory: X's, or those of its transpose
    const bool tall = in.sj != 1;
    const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0, rows = tall ? in.n : in.m, cols = tall ? in.m : in.n;
    const T* g = in.x + b * in.batch;
    const int64_t stride = tall ? in.sj : in.si;
    f16* hi = reinterpret_cast<f16*>(tiles[0]);
    f16* lo = reinterpret_cast<f16*>(tiles[1]);
#pragma unroll
    for (int q = threadIdx.x; q < 64 * 64 / V; q += 256) {
        const int r = q / (64 / V), k0 = q % (64 / V) * V;
        float v[V] = {};
        if (r0 + r < rows) load_row<T>(g + (r0 + r) * stride, c0 + k0, cols, 0.0f, v);
#pragma unroll
        for (int k = 0; k < V; ++k) split(ldexpf(v[k], scale - e), hi[r * kRow + k0 + k], lo[r * kRow + k0 + k]);
    }
    __syncthreads();
    const Planes straight = tall ? xt : x, turned = tall ? x : xt;
    // the lower plane of 16-bit values is zero, and not read in the first step
    constexpr int kPlanes = sizeof(T) > 2 ? 2 : 1;
#pragma unroll
    for (int q = threadIdx.x; q < 64 * 8; q += 256) {
        const int r = q / 8, p = q % 8 * 8;
        const int64_t at = b * straight.batch + (int64_t)(r0 + r) * straight.ld + c0 + p;
        // neighbouring lanes take neighbouring rows of the turned tile, whose columns then share banks less
        const int tr = q % 64, tp = q / 64 * 8;
        const int64_t att = b * turned.batch + (int64_t)(c0 + tr) * turned.ld + r0 + tp;
#pragma unroll
        for (int plane = 0; plane < kPlanes; ++plane) {
            const f16* tile = plane ? lo : hi;
            *reinterpret_cast<half8*>((plane ? straight.lo : straight.hi) + at) =
                *reinterpret_cast<const half8*>(tile + r * kRow + p);
            half8 t;
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = tile[(tp + k) * kRow + tr];
            *reinterpret_cast<half8*>((plane ? turned.lo : turned.hi) + att) = t;
        }
    }
}

// Symmetric: A = X X', the polynomial in A. The others: X times one of these, and the last of them, which
// goes to the caller.
enum class Product { kGram, kPolynomial, kUpdate, kLast };

constexpr bool is_symmetric(Product p) { return p == Product::kGram || p == Product::kPolynomial; }

template <typename T>
struct Output {
    T* x;
    int64_t batch, si, sj;
    int m, n;
};

// How a square tile of a product is computed: its side, the rows and columns of waves that share it, and the
// values of the summed index in one stage of local memory, of which two lie there. Rates measured with both
// operands in two planes, on 2048 x 8192 from 2048 and on 2048 x 2048 from 2048: tiles of 256 1125 and
// 370 TFLOP/s (64 tiles for 256 CUs), of 128 860 and 860, of 64 530 and 574. Larger tiles read less of the
// operands again; a longer stage saves barriers. Tiles of 64 serve products too small to fill the GPU:
// with at most one for each CU (k64Few) 16 waves and stages of 128 measured 10.4 us on 135 tiles from 768, 4
// waves and stages of 64 12.6; with more the latter, of which a CU holds two, 185 us against 223 for
// eight matrices of 512 x 512. Three or four stages were no faster than two, and operands straight to
// registers, each wave on every fourth part of the summed index, half as slow again.
enum class Tile { k256, k128, k64, k64Few };

template <Tile TILE>
struct Shape;
template <>
struct Shape<Tile::k256> {
    static constexpr int kSide = 256, kRows = 2, kCols = 4, kDepth = 32;
};
template <>
struct Shape<Tile::k128> {
    static constexpr int kSide = 128, kRows = 2, kCols = 2, kDepth = 64;
};
template <>
struct Shape<Tile::k64> {
    static constexpr int kSide = 64, kRows = 2, kCols = 2, kDepth = 64;
};
template <>
struct Shape<Tile::k64Few> {
    static constexpr int kSide = 64, kRows = 4, kCols = 4, kDepth = 128;
};
template <Tile TILE>
constexpr int kThreadsOf = Shape<TILE>::kRows * Shape<TILE>::kCols * 64;

// Where a stage holds 16-byte piece p of a row of DEPTH values: pieces are permuted within their row so
// that the 16 lanes that read one piece of 16 rows, and any 8 of them in order, meet different banks.
template <int DEPTH>
__device__ __forceinline__ int piece_of(int row, int p) {
    if constexpr (DEPTH == 32) return p ^ ((row >> 1 & 3) ^ (row >> 3 & 1));
    if constexpr (DEPTH == 128) return p ^ (row & 15);
    return p ^ ((row & 7) ^ (row >> 3 & 1));
}

// 16 bytes a lane straight from memory to local memory, a wave's lanes one after another.
__device__ __forceinline__ void copy_to_local(const f16* from, half8* to) {
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)from,
        (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

struct Operands {
    Planes l, r;     // C = L R': L's rows are C's rows, R's rows its columns
    int depth;       // the summed index, a multiple of 64
    int rows, cols;  // tiles of C
    Planes c, ct;    // C and its transpose
    float factor;    // of the sums, from the scales of both operands to that of C
    Planes own;      // what the sums join: A in the polynomial, X in an update; no lower plane: it is zero
    Coefficients k;
    const Start* start;  // of each matrix
    int before, after;   // what the steps raise X by; before < 0: the first one, whose coefficients are start's
    int exponent;        // from X as stored to the caller's values
    float last;
};

// A step's coefficients for one matrix, and what it is still held too large by after it.
__device__ __forceinline__ Coefficients coefficients_of(const Operands& o, int64_t b, int& left) {
    const Start s = o.start[b];
    left = shift_left(s.shift, o.after);
    return o.before < 0 ? s.k : shifted(o.k, s.shift, o.before, o.after);
}

// A workgroup's tile: the sums over values d0 .. d1 of the summed index of rows i0 of L and j0 of R; d1 - d0 is a
// multiple of 64, and a last stage of 128 may be half one. LP and RP: the planes that are not zero. While the
// waves multiply one stage of the operands the next one is on its way into the other half of local
// memory, so a stage has one barrier. The small terms join the large ones' sums: sums of their own would take
// the error from 0.6 to 0.4 times that of fp32 products, and 5% more time at 2048 x 8192.
template <Tile TILE, int LP, int RP, int MI, int NI>
__device__ __forceinline__ void multiply(const Operands& o, int64_t b, int i0, int j0, int d0, int d1,
                                         half8* stages, float4v (&acc)[MI][NI]) {
    using S = Shape<TILE>;
    constexpr int kThreads = kThreadsOf<TILE>, kDepth = S::kDepth, kPieces = kDepth / 8;
    constexpr int kPlane = S::kSide * kPieces, kStage = (LP + RP) * kPlane;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wi = wave / S::kCols * (MI * 16), wj = wave % S::kCols * (NI * 16);
    const f16* lsrc[2] = {o.l.hi + b * o.l.batch + (int64_t)i0 * o.l.ld,
                          o.l.lo + b * o.l.batch + (int64_t)i0 * o.l.ld};
    const f16* rsrc[2] = {o.r.hi + b * o.r.batch + (int64_t)j0 * o.r.ld,
                          o.r.lo + b * o.r.batch + (int64_t)j0 * o.r.ld};
    const auto load = [&](int d, int part) {
        half8* stage = stages + part * kStage;
#pragma unroll
        for (int p = 0; p < LP + RP; ++p) {
            const bool left = p < LP;
            const f16* src = left ? lsrc[p] : rsrc[p - LP];
            const int64_t ld = left ? o.l.ld : o.r.ld;
#pragma unroll
            for (int q0 = 0; q0 < kPlane; q0 += kThreads) {
                const int q = q0 + threadIdx.x, row = q / kPieces, at = piece_of<kDepth>(row, q % kPieces) * 8;
                if (kDepth <= 64 || d + at < d1)
                    copy_to_local(src + row * ld + d + at, stage + p * kPlane + q0 + wave * 64);
            }
        }
    };
    load(d0, 0);
    for (int d = d0, part = 0; d < d1; d += kDepth, part ^= 1) {
        // this stage has arrived, and every wave has read the other half
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (d + kDepth < d1) load(d + kDepth, part ^ 1);
        const half8* stage = stages + part * kStage;
#pragma unroll
        for (int kk = 0; kk < kPieces / 4; ++kk) {
            if (kDepth > 64 && d + kk * 32 >= d1) break;
            half8 l[LP][MI], r[RP][NI];
#pragma unroll
            for (int p = 0; p < LP; ++p)
#pragma unroll
                for (int x = 0; x < MI; ++x) {
                    const int row = wi + x * 16 + lane % 16;
                    l[p][x] = stage[p * kPlane + row * kPieces + piece_of<kDepth>(row, kk * 4 + lane / 16)];
                }
#pragma unroll
            for (int p = 0; p < RP; ++p)
#pragma unroll
                for (int y = 0; y < NI; ++y) {
                    const int row = wj + y * 16 + lane % 16;
                    r[p][y] = stage[(LP + p) * kPlane + row * kPieces +
                                    piece_of<kDepth>(row, kk * 4 + lane / 16)];
                }
            // R first: a lane then holds four consecutive columns of one row
#pragma unroll
            for (int pl = 0; pl < LP; ++pl)
#pragma unroll
                for (int pr = 0; pr < (pl ? 1 : RP); ++pr)
#pragma unroll
                    for (int x = 0; x < MI; ++x)
#pragma unroll
                        for (int y = 0; y < NI; ++y)
                            acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[pr][y], l[pl][x], acc[x][y], 0, 0, 0);
        }
    }
}

// Tells the compiler that local memory was written for other lanes of the wave, whose accesses the
// hardware keeps in order.
__device__ __forceinline__ void wave_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// Local memory of a wave in which 16 columns of its part of C turn round: 16 rows of both planes.
template <int MI>
constexpr int kTurnRow = MI * 16 + 8;  // values; the 8 shift the rows' banks
template <int MI>
constexpr int kTurn = 2 * 16 * kTurnRow<MI>;

// MI tiles of 16 x 16 one below the other, from row i (the lane's own) and column j (its first of four) on: what
// the product is for, and its places. `mirrored`: in C's transpose too, through the wave's `turn`.
template <Product KIND, int MI, typename T>
__device__ __forceinline__ void finish(const Operands& o, const Output<T>& out, int64_t b, Coefficients k,
                                       int left, int i, int j, bool mirrored, const float4v (&sum)[MI], f16* turn) {
    const int lane = threadIdx.x % 64;
    half4 own[MI], low[MI] = {};  // all on their way before the first store
    if constexpr (KIND != Product::kGram) {
#pragma unroll
        for (int x = 0; x < MI; ++x) {
            const int64_t at = b * o.own.batch + (int64_t)(i + x * 16) * o.own.ld + j;
            own[x] = *reinterpret_cast<const half4*>(o.own.hi + at);
            if (o.own.lo) low[x] = *reinterpret_cast<const half4*>(o.own.lo + at);
        }
    }
#pragma unroll
    for (int x = 0; x < MI; ++x) {
        const int row = i + x * 16;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (KIND == Product::kGram) v[q] = sum[x][q] * o.factor;
            else if constexpr (KIND == Product::kPolynomial)
                v[q] = k.b * ((float)own[x][q] + (float)low[x][q]) + k.c * sum[x][q];
            else v[q] = __builtin_fmaf(k.a, (float)own[x][q] + (float)low[x][q], sum[x][q] * o.factor);
            if constexpr (KIND == Product::kLast) v[q] = ldexpf(v[q], o.exponent - left) * o.last;
        }
        if constexpr (KIND == Product::kLast) {
            T* to = out.x + b * out.batch + row * out.si + j * out.sj;
            if (out.sj == 1 && row < out.m && j + 4 <= out.n) {
                typedef T U __attribute__((ext_vector_type(4), aligned(sizeof(T))));
                U u;
#pragma unroll
                for (int q = 0; q < 4; ++q) u[q] = (T)v[q];
                *reinterpret_cast<U*>(to) = u;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (row < out.m && j + q < out.n) to[q * out.sj] = (T)v[q];
            }
        } else {
            half4 h, w;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f16 hi, lo;
                split(v[q], hi, lo);
                h[q] = hi;
                w[q] = lo;
            }
            const int64_t at = b * o.c.batch + (int64_t)row * o.c.ld + j;
            *reinterpret_cast<half4*>(o.c.hi + at) = h;
            *reinterpret_cast<half4*>(o.c.lo + at) = w;
            if (mirrored) {
                f16* to = turn + (lane / 16 * 4) * kTurnRow<MI> + x * 16 + lane % 16;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    to[q * kTurnRow<MI>] = h[q];
                    to[(16 + q) * kTurnRow<MI>] = w[q];
                }
            }
        }
    }
    if constexpr (KIND != Product::kLast) {
        if (mirrored) {
            wave_order();
            const int i0 = i - lane % 16, j0 = j - lane / 16 * 4;
            constexpr int kRowPieces = MI * 2;
#pragma unroll
            for (int q = 0; q < kRowPieces * 16; q += 64) {
                const int row = (q + lane) / kRowPieces, p = (q + lane) % kRowPieces * 8;
                const int64_t att = b * o.ct.batch + (int64_t)(j0 + row) * o.ct.ld + i0 + p;
                if (q + lane < kRowPieces * 16) {
                    *reinterpret_cast<half8*>(o.ct.hi + att) =
                        *reinterpret_cast<const half8*>(turn + row * kTurnRow<MI> + p);
                    *reinterpret_cast<half8*>(o.ct.lo + att) =
                        *reinterpret_cast<const half8*>(turn + (16 + row) * kTurnRow<MI> + p);
                }
            }
            wave_order();
        }
    }
}

// Tile t of the tiles on and above the diagonal, column by column: its row is ti <= tj.
__device__ __forceinline__ void triangle(int t, int& ti, int& tj) {
    tj = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
    while (tj * (tj + 1) / 2 > t) --tj;
    ti = t - tj * (tj + 1) / 2;
}

// C = L R', a workgroup a tile. Bound by the MFMA rate and what each stage waits for, and in an update by X's way to
// memory and back: a X + P X at 2048 x 8192 takes 239 us with three products (2.1e11 flop, 0.86 PFLOP/s), 206 where
// it goes to the caller alone (1.0), and 168 with two products, from X0 in 16 bits (0.82). With too few tiles latency does: 11 us for A of three matrices of 515 x 770, 135 tiles.
template <Product KIND, Tile TILE, int LP, int RP, typename T>
__global__ __launch_bounds__(kThreadsOf<TILE>) void product_kernel(Operands o, Output<T> out) {
    using S = Shape<TILE>;
    constexpr bool kSymmetric = is_symmetric(KIND);
    constexpr int MI = S::kSide / S::kRows / 16, NI = S::kSide / S::kCols / 16;
    extern __shared__ half8 stages[];
    // one XCD's workgroups take neighbouring tiles: all rows of some columns
    const int tiles = kSymmetric ? o.rows * (o.rows + 1) / 2 : o.rows * o.cols;
    const int all = xcd_contiguous(blockIdx.x, gridDim.x);
    const int64_t b = all / tiles;
    const int tile = all % tiles;
    int ti = tile % o.rows, tj = tile / o.rows;
    if constexpr (kSymmetric) triangle(tile, ti, tj);
    float4v acc[MI][NI] = {};
    multiply<TILE, LP, RP>(o, b, ti * S::kSide, tj * S::kSide, 0, o.depth, stages, acc);
    Coefficients k = {};
    int left = 0;
    if (KIND != Product::kGram) k = coefficients_of(o, b, left);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int i = ti * S::kSide + wave / S::kCols * (MI * 16) + lane % 16;
    const int j = tj * S::kSide + wave % S::kCols * (NI * 16) + lane / 16 * 4;
    static_assert(KIND == Product::kLast ||
                      S::kRows * S::kCols * kTurn<MI> <= 2 * (LP + RP) * S::kSide * S::kDepth,
                  "the waves' turns fit into the stages");
    if constexpr (KIND != Product::kLast) __syncthreads();  // every wave has read the last stage
    f16* turn = reinterpret_cast<f16*>(stages) + wave * kTurn<MI>;
#pragma unroll
    for (int y = 0; y < NI; ++y) {
        float4v column[MI];
#pragma unroll
        for (int x = 0; x < MI; ++x) column[x] = acc[x][y];
        finish<KIND, MI, T>(o, out, b, k, left, i, j + y * 16, !kSymmetric || ti != tj, column, turn);
    }
}

// A symmetric product whose tiles fill the GPU badly: workgroups share all stages of all tiles evenly, in
// order, and leave each part of a tile's sum in memory, in the order of the registers; the part of
// worker w in tile t is part t + w. 38 us for a product of 2048 x 2048 from 2048 (136 tiles, 2.7e10 flop, 0.72
// PFLOP/s) and 11 to join its parts, 15 where the polynomial reads A as well.
struct Shares {
    float* parts;
    int stages;   // of 64 values of the summed index, of all tiles
    int depth;    // those of a tile
    int workers;  // as many as there are stages, or fewer
    __device__ __forceinline__ int begin(int w) const {
        return (int)((uint64_t)(uint32_t)w * (uint32_t)stages / (uint32_t)workers);
    }
    // The worker that holds a stage.
    __device__ __forceinline__ int holder(int stage) const {
        int w = (int)((float)stage * ((float)workers / (float)stages));
        while (w > 0 && begin(w) > stage) --w;
        while (begin(w + 1) <= stage) ++w;
        return w;
    }
};

template <Tile TILE, int LP, int RP>
__global__ __launch_bounds__(kThreadsOf<TILE>) void shared_product_kernel(Operands o, Shares s) {
    using S = Shape<TILE>;
    constexpr int MI = S::kSide / S::kRows / 16, NI = S::kSide / S::kCols / 16, kThreads = kThreadsOf<TILE>;
    extern __shared__ half8 stages[];
    const int tiles = o.rows * (o.rows + 1) / 2;
    const int w = xcd_contiguous(blockIdx.x, s.workers);
    const int end = s.begin(w + 1);
    for (int at = s.begin(w); at < end;) {
        const int t = at / s.depth;
        const int stop = (t + 1) * s.depth < end ? (t + 1) * s.depth : end;
        int ti, tj;
        triangle(t % tiles, ti, tj);
        float4v acc[MI][NI] = {};
        multiply<TILE, LP, RP>(o, t / tiles, ti * S::kSide, tj * S::kSide, (at - t * s.depth) * 64,
                                             (stop - t * s.depth) * 64, stages, acc);
        float* part = s.parts + (int64_t)(t + w) * (S::kSide * S::kSide) + threadIdx.x * 4;
#pragma unroll
        for (int x = 0; x < MI; ++x)
#pragma unroll
            for (int y = 0; y < NI; ++y)
                *reinterpret_cast<float4v*>(part + (y * MI + x) * (kThreads * 4)) = acc[x][y];
        at = stop;
        __syncthreads();  // every wave has read the last stage
    }
}

// The parts of a tile, added in the workers' order: a workgroup takes 16 columns of each wave's part of C.
template <Product KIND, Tile TILE>
__global__ __launch_bounds__(kThreadsOf<TILE>) void join_product_kernel(Operands o, Shares s) {
    using S = Shape<TILE>;
    constexpr int MI = S::kSide / S::kRows / 16, NI = S::kSide / S::kCols / 16, kThreads = kThreadsOf<TILE>;
    __shared__ half8 turns[kThreads / 64 * kTurn<MI> / 8];
    const int tiles = o.rows * (o.rows + 1) / 2;
    const int t = blockIdx.x / NI, y = blockIdx.x % NI;
    const int64_t b = t / tiles;
    int ti, tj;
    triangle(t % tiles, ti, tj);
    const int w0 = s.holder(t * s.depth), w1 = s.holder((t + 1) * s.depth - 1);
    const float* part = s.parts + (int64_t)t * (S::kSide * S::kSide) + y * (MI * kThreads * 4) + threadIdx.x * 4;
    float4v sum[MI] = {};
    constexpr int kAtOnce = 3;  // workers whose parts are on their way together
    for (int w = w0; w <= w1; w += kAtOnce) {
        float4v v[kAtOnce][MI];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int from = w + q <= w1 ? w + q : w1;
#pragma unroll
            for (int x = 0; x < MI; ++x)
                v[q][x] = *reinterpret_cast<const float4v*>(part + (int64_t)from * (S::kSide * S::kSide) + x * (kThreads * 4));
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q)
            if (w + q <= w1) {
#pragma unroll
                for (int x = 0; x < MI; ++x) sum[x] += v[q][x];
            }
    }
    Coefficients k = {};
    int left = 0;
    if (KIND != Product::kGram) k = coefficients_of(o, b, left);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    finish<KIND, MI>(o, Output<f16>{}, b, k, left, ti * S::kSide + wave / S::kCols * (MI * 16) + lane % 16,
                     tj * S::kSide + wave % S::kCols * (NI * 16) + y * 16 + lane / 16 * 4, ti != tj, sum,
                     reinterpret_cast<f16*>(turns) + wave * kTurn<MI>);
}

// Whole matrices of up to 64 x 256 in one workgroup each, with everything in local memory: X both ways
// round, A and P, 160 KiB at the largest. The product kernels would take three launches a step of 4 us each,
// whatever they compute. Instructions bound it, so a lane's places in the permuted rows are worked out
// once: rows of a tile start at multiples of 16, and what a permutation takes from them is the lane's own. Five
// steps of 64 x 256 take 41 us.
constexpr int kSmallThreads = 1024;

struct SmallSteps {
    int steps;
    Coefficients k[kMaxSteps];
    int grown[kMaxSteps + 1];  // before each step, and after the last
};

// From sums of products to what is stored, and to the caller's values.
struct SmallFactors {
    int x;  // the exponent of X's scale
    float gram, update;
    int exponent;  // from X as stored to the caller's values
    float last;
};

// Matrices in local memory lie in panels of 64 columns: 8 pieces a row, permuted as a stage's.
struct LocalPlanes {
    half8 *hi, *lo;
    int panel;  // pieces from one panel to the next
};

__device__ __forceinline__ int permuted(int row, int p) { return piece_of<64>(row, p); }

// A lane's operands of a tile: its row's piece of each half of a panel, from the tile's first row on.
struct LaneOffsets {
    int half[2];    // operands
    int row, flip;  // a value's row and its permutation, as C holds it: four columns of one row
    int column;     // of the first of the four, 0 to 12
    __device__ __forceinline__ explicit LaneOffsets(int lane) {
        const int r = lane % 16;
        half[0] = r * 8 + permuted(r, lane / 16);
        half[1] = r * 8 + permuted(r, 4 + lane / 16);
        row = r;
        flip = permuted(r, 0);
        column = lane / 16 * 4;
    }
};

// acc += the 16 x 16 tiles of L R' for NL tiles of rows from L's row i on (every 16) and R's 16 rows from j on,
// over one panel; the small terms go into `cross`, which may be `acc` where registers are short.
template <int NL>
__device__ __forceinline__ void local_product(LocalPlanes l, int i, LocalPlanes r, int j, int panel,
                                              const LaneOffsets& at, float4v (&acc)[NL], float4v (&cross)[NL]) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        const int rr = panel * r.panel + j * 8 + at.half[kk];
        const half8 rh = r.hi[rr], rl = r.lo[rr];
#pragma unroll
        for (int x = 0; x < NL; ++x) {
            const int ll = panel * l.panel + (i + x * 16) * 8 + at.half[kk];
            const half8 lh = l.hi[ll], lw = l.lo[ll];
            acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rh, lh, acc[x], 0, 0, 0);
            cross[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rl, lh, cross[x], 0, 0, 0);
            cross[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rh, lw, cross[x], 0, 0, 0);
        }
    }
}

// The tile at row i and column j (multiples of 16) of a matrix, and with `t` of its transpose.
__device__ __forceinline__ void local_store(LocalPlanes m, const LocalPlanes* t, int i, int j,
                                            const LaneOffsets& at, const float (&v)[4]) {
    half4 h, w;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f16 hi, lo;
        split(v[q], hi, lo);
        h[q] = hi;
        w[q] = lo;
    }
    const int to = (j / 64 * m.panel + (i + at.row) * 8 + ((j % 64 + at.column) / 8 ^ at.flip)) * 8 + at.column % 8;
    *reinterpret_cast<half4*>(reinterpret_cast<f16*>(m.hi) + to) = h;
    *reinterpret_cast<half4*>(reinterpret_cast<f16*>(m.lo) + to) = w;
    if (t) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = at.column + q;
            const int too = ((j + r) * 8 + ((i + at.row) / 8 ^ permuted(r, 0))) * 8 + at.row % 8;
            reinterpret_cast<f16*>(t->hi)[too] = h[q];
            reinterpret_cast<f16*>(t->lo)[too] = w[q];
        }
    }
}

// The tile's values, each lane its own four.
__device__ __forceinline__ void local_load(LocalPlanes m, int i, int j, const LaneOffsets& at, float (&v)[4]) {
    const int from = (j / 64 * m.panel + (i + at.row) * 8 + ((j % 64 + at.column) / 8 ^ at.flip)) * 8 + at.column % 8;
    const half4 h = *reinterpret_cast<const half4*>(reinterpret_cast<const f16*>(m.hi) + from);
    const half4 w = *reinterpret_cast<const half4*>(reinterpret_cast<const f16*>(m.lo) + from);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = (float)h[q] + (float)w[q];
}

// pieces of X (either way round) and of A or P in one plane
__host__ __device__ constexpr int small_x(int n) { return kSmallSide * n / 8; }
constexpr int kSmallA = kSmallSide * kSmallSide / 8;

// A workgroup's matrices in local memory, for n columns of X (whole panels).
struct SmallLocal {
    LocalPlanes x, xt, a, p;
    __device__ __forceinline__ SmallLocal(half8* local, int n)
        : x{local, local + small_x(n), kSmallA},
          xt{local + 2 * small_x(n), local + 3 * small_x(n), 0},
          a{local + 4 * small_x(n), local + 4 * small_x(n) + kSmallA, 0},
          p{local + 4 * small_x(n) + 2 * kSmallA, local + 4 * small_x(n) + 3 * kSmallA, 0} {}
};

// Its columns of G, from j0 on, in registers: vectors as they lie in memory, with X's rows or columns.
constexpr int kSmallMine = kSmallSide * kSmallLong / kSmallThreads;

template <typename T>
__device__ __forceinline__ void small_fetch(const Input<T>& in, int64_t b, int j0, float (&v)[kSmallMine / kVec<T>][kVec<T>]) {
    constexpr int V = kVec<T>;
    const bool tall = in.sj != 1;
    const T* g = in.x + b * in.batch;
#pragma unroll
    for (int q = 0; q < kSmallMine / V; ++q) {
        const int e = q * kSmallThreads + threadIdx.x;
        const int r = tall ? e / (kSmallSide / V) : e / (kSmallLong / V);
        const int c = tall ? e % (kSmallSide / V) * V : e % (kSmallLong / V) * V;
#pragma unroll
        for (int k = 0; k < V; ++k) v[q][k] = 0.0f;
        if (tall && j0 + r < in.n) load_row<T>(g + (int64_t)(j0 + r) * in.sj, c, in.m, 0.0f, v[q]);
        if (!tall && r < in.m) load_row<T>(g + (int64_t)r * in.si, j0 + c, in.n, 0.0f, v[q]);
    }
}

// Scaled and split into X, both ways round.
template <int V>
__device__ __forceinline__ void small_split(const SmallLocal& m, bool tall, int n, int exponent,
                                            const float (&v)[kSmallMine / V][V]) {
    typedef f16 halfv __attribute__((ext_vector_type(V)));
    const LocalPlanes straight = tall ? m.xt : m.x, turned = tall ? m.x : m.xt;
#pragma unroll
    for (int q = 0; q < kSmallMine / V; ++q) {
        const int e = q * kSmallThreads + threadIdx.x;
        const int r = tall ? e / (kSmallSide / V) : e / (kSmallLong / V);
        const int c = tall ? e % (kSmallSide / V) * V : e % (kSmallLong / V) * V;
        if ((tall ? r : c) >= n) continue;
        halfv h, w;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            f16 hi, lo;
            split(ldexpf(v[q][k], exponent), hi, lo);
            h[k] = hi;
            w[k] = lo;
        }
        const int to = (c / 64 * straight.panel + r * 8 + permuted(r, c % 64 / 8)) * 8 + c % 8;
        *reinterpret_cast<halfv*>(reinterpret_cast<f16*>(straight.hi) + to) = h;
        *reinterpret_cast<halfv*>(reinterpret_cast<f16*>(straight.lo) + to) = w;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int too = (r / 64 * turned.panel + (c + k) * 8 + permuted(c + k, r % 64 / 8)) * 8 + r % 8;
            reinterpret_cast<f16*>(turned.hi)[too] = h[k];
            reinterpret_cast<f16*>(turned.lo)[too] = w[k];
        }
    }
}

// The wave's tile of A over the workgroup's columns, as sums of stored values.
__device__ __forceinline__ float4v small_gram(const SmallLocal& m, int n, int ti, int tj, const LaneOffsets& at) {
    float4v acc[1] = {}, cross[1] = {};
    for (int q = 0; q < n / 64; ++q) local_product<1>(m.x, ti, m.x, tj, q, at, acc, cross);
    return acc[0] + cross[0];
}

// From the wave's tile of A to its tile of P in local memory, for everyone.
__device__ __forceinline__ void small_polynomial(const SmallLocal& m, float4v a, Coefficients k, float factor, int ti,
                                                 int tj, const LaneOffsets& at) {
    float gram[4], poly[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) gram[c] = a[c] * factor;
    local_store(m.a, nullptr, ti, tj, at, gram);
    __syncthreads();
    float4v acc[1] = {}, cross[1] = {};
    local_product<1>(m.a, ti, m.a, tj, 0, at, acc, cross);
    acc[0] += cross[0];
#pragma unroll
    for (int c = 0; c < 4; ++c)
        poly[c] = k.b * gram[c] + k.c * acc[0][c];
    local_store(m.p, nullptr, ti, tj, at, poly);
    __syncthreads();
}

// X <- a X + P X in local memory, or with `last` to the caller, whose columns begin at j0.
template <typename T>
__device__ __forceinline__ void small_update(const SmallLocal& m, int n, int col, float a, const LaneOffsets& at, bool last,
                                             int left, const Output<T>& out, int64_t b, int j0, SmallFactors f) {
    constexpr int kTiles = kSmallSide / 16;
    float4v next[kTiles] = {};
    if (col < n) local_product<kTiles>(m.p, 0, m.xt, col, 0, at, next, next);
    __syncthreads();
    if (col < n) {
#pragma unroll
        for (int y = 0; y < kTiles; ++y) {
            float w[4];
            local_load(m.x, y * 16, col, at, w);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                w[c] = __builtin_fmaf(a, w[c], next[y][c] * f.update);
                if (last) w[c] = ldexpf(w[c], f.exponent - left) * f.last;
            }
            if (!last) {
                local_store(m.x, &m.xt, y * 16, col, at, w);
                continue;
            }
            const int i = y * 16 + at.row, j = j0 + col + at.column;
            if (i < out.m) {
                T* to = out.x + b * out.batch + i * out.si + j * out.sj;
                if (out.sj == 1) {
                    store_row<T, 4>(to, 0, out.n - j, w);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (j + c < out.n) to[c * out.sj] = (T)w[c];
                }
            }
        }
    }
    __syncthreads();
}

// n: X's columns padded to whole panels.
template <typename T>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(Input<T> in, Output<T> out, int n, SmallSteps s,
                                                              SmallFactors f, double eps) {
    extern __shared__ half8 local[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    constexpr int kWaves = kSmallThreads / 64, kTiles = kSmallSide / 16;
    static_assert(kTiles * kTiles == kWaves && kSmallLong / 16 == kWaves, "a tile of A, a column of X a wave");
    const SmallLocal m(local, n);
    const LaneOffsets at(lane);
    float v[kSmallMine / kVec<T>][kVec<T>];
    small_fetch(in, blockIdx.x, 0, v);
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < kSmallMine / kVec<T>; ++q)
#pragma unroll
        for (int c = 0; c < kVec<T>; ++c) sum += (double)v[q][c] * (double)v[q][c];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    double* sums = reinterpret_cast<double*>(m.p.hi);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sums[w];
    int e;
    Start start;
    scale_of(sum, s.k[0], eps, s.grown[1], e, start);
    small_split<kVec<T>>(m, in.sj != 1, n, f.x - e, v);
    __syncthreads();
    const int ti = wave / kTiles * 16, tj = wave % kTiles * 16;  // the wave's tile of A and P
    for (int step = 0; step < s.steps; ++step) {
        const Coefficients k =
            step == 0 ? start.k : shifted(s.k[step], start.shift, s.grown[step], s.grown[step + 1]);
        small_polynomial(m, small_gram(m, n, ti, tj, at), k, f.gram, ti, tj, at);
        small_update(m, n, wave * 16, k.a, at, step + 1 == s.steps, shift_left(start.shift, s.grown[step + 1]), out,
                     blockIdx.x, 0, f);
    }
}

// Matrices of up to 64 rows and some thousand columns: strips of 256 columns, each with a workgroup that keeps
// it as the one above does, and one launch a step. What a step needs of the other strips is their part of
// A, which they left in memory in the launch before; every workgroup adds all parts in order and
// forms P for itself. Latency bounds it. 64 x 2048 takes 66 us, and 149 with the product kernels, whose only tile of A runs
// through 2048 columns on one CU.
struct Strips {
    float* parts;  // [batch][strips][64 x 64], in the order of the registers: read; `made`: written
    float* made;
    half8* planes;  // [batch][strips]: X of a strip as in local memory
    int strips;
};

constexpr int kStripPlanes = 4 * small_x(kSmallLong);  // pieces

template <typename T>
__global__ __launch_bounds__(kSmallThreads) void strip_start_kernel(Input<T> in, const double* norm, int nparts,
                                                                    int scale, Coefficients k, double eps, int grown,
                                                                    Strips s, Start* start) {
    extern __shared__ half8 local[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t b = blockIdx.y, strip = b * s.strips + blockIdx.x;
    const SmallLocal m(local, kSmallLong);
    const LaneOffsets at(lane);
    float v[kSmallMine / kVec<T>][kVec<T>];
    small_fetch(in, b, blockIdx.x * kSmallLong, v);
    double sum = 0.0;
    for (int i = lane; i < nparts; i += 64) sum += norm[b * kNormParts + i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    int e;
    Start mine;
    scale_of(sum, k, eps, grown, e, mine);
    if (blockIdx.x == 0 && threadIdx.x == 0) start[b] = mine;
    small_split<kVec<T>>(m, in.sj != 1, kSmallLong, scale - e, v);
    __syncthreads();
    const float4v a = small_gram(m, kSmallLong, wave / 4 * 16, wave % 4 * 16, at);
    reinterpret_cast<float4v*>(s.made)[strip * kSmallThreads + threadIdx.x] = a;
#pragma unroll
    for (int q = 0; q < kStripPlanes; q += kSmallThreads)
        s.planes[strip * kStripPlanes + q + threadIdx.x] = local[q + threadIdx.x];
}

template <typename T>
__global__ __launch_bounds__(kSmallThreads) void strip_step_kernel(Output<T> out, Strips s, Coefficients k,
                                                                   const Start* start, int before, int after,
                                                                   bool last, SmallFactors f) {
    extern __shared__ half8 local[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t b = blockIdx.y, strip = b * s.strips + blockIdx.x;
    const SmallLocal m(local, kSmallLong);
    const LaneOffsets at(lane);
#pragma unroll
    for (int q = 0; q < kStripPlanes; q += kSmallThreads)
        local[q + threadIdx.x] = s.planes[strip * kStripPlanes + q + threadIdx.x];
    const float4v* parts = reinterpret_cast<const float4v*>(s.parts) + b * s.strips * kSmallThreads + threadIdx.x;
    float4v a = {};
#pragma unroll 8
    for (int q = 0; q < s.strips; ++q) a += parts[q * kSmallThreads];
    const Start mine = start[b];
    k = before < 0 ? mine.k : shifted(k, mine.shift, before, after);
    const int ti = wave / 4 * 16, tj = wave % 4 * 16;
    small_polynomial(m, a, k, f.gram, ti, tj, at);
    small_update(m, kSmallLong, wave * 16, k.a, at, last, shift_left(mine.shift, after), out, b, blockIdx.x * kSmallLong, f);
    if (last) return;
    a = small_gram(m, kSmallLong, ti, tj, at);
    reinterpret_cast<float4v*>(s.made)[strip * kSmallThreads + threadIdx.x] = a;
#pragma unroll
    for (int q = 0; q < kStripPlanes; q += kSmallThreads)
        s.planes[strip * kStripPlanes + q + threadIdx.x] = local[q + threadIdx.x];
}

// The workspace: norm parts and what each matrix starts from, then the planes of X and X' twice, of A and P, and the parts
// of products that are shared.
struct Layout {
    int64_t parts, start, x[2], xt[2], a, p, shares, bytes;  // byte offsets
    int64_t strip_parts[2], strip_planes;
    int64_t m, n;
    Tiles tiles;
    bool small;   // nothing else then
    int strips;   // 0: the product kernels; otherwise norm, start and strips only
};

Layout layout_of(int64_t batch, int64_t rows, int64_t cols) {
    Layout w;
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    w.small = m <= kSmallSide && n <= kSmallLong;
    w.m = m;
    w.n = n;
    w.bytes = 0;
    w.strips = 0;
    if (w.small) return w;
    if (m <= kSmallSide && n <= kSmallLong * kMostStrips) w.strips = (int)padded(n, kSmallLong) / kSmallLong;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    w.parts = take(batch * kNormParts * (int64_t)sizeof(double));
    w.start = take(batch * (int64_t)sizeof(Start));
    if (w.strips) {
        for (int64_t& p : w.strip_parts) p = take(batch * w.strips * kSmallSide * kSmallSide * (int64_t)sizeof(float));
        w.strip_planes = take(batch * w.strips * kStripPlanes * (int64_t)sizeof(half8));
        w.bytes = at + 256;
        return w;
    }
    w.tiles = tiles_of(batch, m, n);
    const int64_t pm = padded(m, w.tiles.pad()), pn = padded(n, w.tiles.pad());
    const int64_t xs = batch * pm * pn * 2 * (int64_t)sizeof(f16), as = batch * pm * pm * 2 * (int64_t)sizeof(f16);
    for (int i = 0; i < 2; ++i) {
        w.x[i] = take(xs);
        w.xt[i] = take(xs);
    }
    w.a = take(as);
    w.p = take(as);
    int64_t most = 0;
    for (const int64_t depth : {pn, pm}) {
        const ProductForm f = form_of(batch, pm, pm, depth, w.tiles.symmetric, true);
        const int64_t bytes = f.workers ? (f.tiles + f.workers) * f.tile * f.tile * (int64_t)sizeof(float) : 0;
        most = bytes > most ? bytes : most;
    }
    w.shares = take(most);
    w.bytes = at + 256;
    return w;
}

template <typename K>
bool allow_local(K kernel, size_t local) {
    return local <= 65536 ||
           hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)local) == hipSuccess;
}

template <Product KIND, Tile TILE, int LP, int RP, typename T>
int launch_product(const Operands& o, const Output<T>& out, const ProductForm& form, float* parts, hipStream_t stream) {
    using S = Shape<TILE>;
    constexpr size_t local = (size_t)2 * (LP + RP) * S::kSide * S::kDepth * sizeof(f16);
    if constexpr (is_symmetric(KIND)) {
        if (form.workers) {
            const auto kernel = shared_product_kernel<TILE, LP, RP>;
            if (!allow_local(kernel, local)) return TRIVANCE_EHIP;
            const Shares s{parts, (int)form.tiles * (o.depth / 64), o.depth / 64, form.workers};
            kernel<<<form.workers, kThreadsOf<TILE>, local, stream>>>(o, s);
            join_product_kernel<KIND, TILE><<<(unsigned)(form.tiles * (S::kSide / S::kCols / 16)), kThreadsOf<TILE>, 0, stream>>>(o, s);
            return launch_status();
        }
    }
    const auto kernel = product_kernel<KIND, TILE, LP, RP, T>;
    if (!allow_local(kernel, local)) return TRIVANCE_EHIP;
    kernel<<<(unsigned)form.tiles, kThreadsOf<TILE>, local, stream>>>(o, out);
    return launch_status();
}

// Which planes a product takes: hi hi + hi lo + lo hi, or kExact: X0 from 16 bits, whose lower plane is zero.
enum class Depth { kBoth, kExact };

// A product by the call's tiles.
template <Product KIND, typename T>
int product(Operands o, const Output<T>& out, int64_t batch, int tile, Depth depth, float* parts,
            hipStream_t stream) {
    const ProductForm form = form_of(batch, o.rows, o.cols, o.depth, tile, is_symmetric(KIND));
    o.rows = o.rows / tile;
    o.cols = o.cols / tile;
#define LAUNCH(TILE, LP, RP) return launch_product<KIND, Tile::TILE, LP, RP>(o, out, form, parts, stream)
#define LAUNCH_SMALLER(LP, RP)              \
    if (tile == 128) LAUNCH(k128, LP, RP);  \
    if (form.few) LAUNCH(k64Few, LP, RP);   \
    LAUNCH(k64, LP, RP)
    if constexpr (KIND == Product::kGram) {
        if (depth == Depth::kExact) {
            LAUNCH_SMALLER(1, 1);
        }
    }
    if constexpr (KIND == Product::kUpdate || (KIND == Product::kLast && sizeof(T) == 2)) {
        if (depth == Depth::kExact) {
            if (tile == 256) LAUNCH(k256, 2, 1);
            LAUNCH_SMALLER(2, 1);
        }
    }
    if constexpr (!is_symmetric(KIND)) {
        if (tile == 256) LAUNCH(k256, 2, 2);
    }
    LAUNCH_SMALLER(2, 2);
#undef LAUNCH_SMALLER
#undef LAUNCH
}

// The ranges that the coefficients give: the largest singular value of X in any step, from values in [0, 1] on,
// and the largest factor that P takes it by, and the powers of two by which X, A and P can be held in fp16.
// The first step's factors may be doubled (what is left of the norm).
struct Ranges {
    bool ok;
    int x, a, p;  // exponents
    int grown[kMaxSteps + 1];  // singular values are raised by 2^grown at most before each step, and after the last
};

Ranges ranges_of(const float* k, int steps) {
    constexpr double kMargin = 1.01;  // between the samples, and the rounding of the products
    double most = 1.0, all = 1.0, factor = 0.0, growth = 0.0;
    Ranges r;
    r.ok = false;
    r.grown[0] = 0;
    for (int s = 0; s < steps; ++s) {
        const double a = k[3 * s], b = k[3 * s + 1], c = k[3 * s + 2];
        double next = 0.0, raised = 1.0;
        constexpr int kSamples = 256;
        for (int i = 0; i <= kSamples; ++i) {
            const double v = most * i / kSamples, p = std::fabs(a + v * v * (b + v * v * c));
            if (!(p <= 15.0)) return r;
            const double f = v * v * std::fabs(b + v * v * c);
            factor = std::fmax(factor, s == 0 ? 2.0 * f : f);
            next = std::fmax(next, p * v);
            raised = std::fmax(raised, p * kMargin);
        }
        growth += std::log2(raised);
        r.grown[s + 1] = (int)std::ceil(growth);
        most = next * kMargin;
        if (!(most <= 3.9)) return r;
        all = std::fmax(all, most);
    }
    factor = std::fmax(factor, 1.0) * kMargin;
    const auto exponent = [](double bound) { return std::ilogb(60000.0 / bound); };
    r.ok = true;
    r.x = exponent(all);
    r.a = exponent(all * all);
    r.p = exponent(factor);
    return r;
}

float power(int exponent) { return std::ldexp(1.0f, exponent); }

template <typename T>
int run(Input<T> in, Output<T> out, int64_t batch, int steps, const float* k, const Ranges& range, float scale,
        double eps, const Layout& w, void* workspace, hipStream_t stream) {
    const auto coefficients = [&](int s) {
        return Coefficients{k[3 * s], k[3 * s + 1] * power(range.p - range.a),
                            k[3 * s + 2] * power(range.p - 2 * range.a)};
    };
    const float gram = power(range.a - 2 * range.x);
    const SmallFactors factors{range.x, gram, power(-range.p), -range.x, scale};
    if (w.small) {
        SmallSteps s;
        s.steps = steps;
        for (int i = 0; i < steps; ++i) s.k[i] = coefficients(i);
        for (int i = 0; i <= steps; ++i) s.grown[i] = range.grown[i];
        const int n = (int)padded(w.n, 64);
        const size_t local = sizeof(half8) * (4 * small_x(n) + 4 * kSmallA);
        if (!allow_local(&small_kernel<T>, local)) return TRIVANCE_EHIP;
        small_kernel<T><<<(unsigned)batch, kSmallThreads, local, stream>>>(in, out, n, s, factors, eps);
        return launch_status();
    }
    char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
    double* parts = reinterpret_cast<double*>(base + w.parts);
    Start* start = reinterpret_cast<Start*>(base + w.start);
    const unsigned nb = (unsigned)batch;
    const int rows = in.sj != 1 ? in.n : in.m;
    const int64_t pieces = (int64_t)rows * (((rows == in.n ? in.m : in.n) + 256 * kVec<T> - 1) / (256 * kVec<T>));
    const int nparts = (int)(pieces < kNormParts ? pieces : kNormParts);
    const Coefficients k0 = coefficients(0);
    norm_parts_kernel<T><<<dim3(nparts, nb), 256, 0, stream>>>(in, parts);
    if (w.strips) {
        const size_t local = sizeof(half8) * (kStripPlanes + 4 * kSmallA);
        if (!allow_local(&strip_start_kernel<T>, local) || !allow_local(&strip_step_kernel<T>, local))
            return TRIVANCE_EHIP;
        Strips s{reinterpret_cast<float*>(base + w.strip_parts[0]), reinterpret_cast<float*>(base + w.strip_parts[1]),
                 reinterpret_cast<half8*>(base + w.strip_planes), w.strips};
        const dim3 grid(w.strips, nb);
        strip_start_kernel<T><<<grid, kSmallThreads, local, stream>>>(in, parts, nparts, range.x, k0, eps, range.grown[1], s,
                                                                        start);
        for (int i = 0; i < steps; ++i) {
            float* read = s.made;
            s.made = s.parts;
            s.parts = read;
            strip_step_kernel<T><<<grid, kSmallThreads, local, stream>>>(
                out, s, coefficients(i), start, i == 0 ? -1 : range.grown[i], range.grown[i + 1], i + 1 == steps, factors);
        }
        return launch_status();
    }
    const Tiles tiles = w.tiles;
    const int m = (int)padded(w.m, tiles.pad()), n = (int)padded(w.n, tiles.pad());
    const auto planes = [&](int64_t offset, int64_t rows, int ld) {
        f16* hi = reinterpret_cast<f16*>(base + offset);
        return Planes{hi, hi + batch * rows * ld, rows * ld, ld};
    };
    float* shares = reinterpret_cast<float*>(base + w.shares);
    Planes x[2], xt[2];
    for (int i = 0; i < 2; ++i) {
        x[i] = planes(w.x[i], m, n);
        xt[i] = planes(w.xt[i], n, m);
    }
    const Planes a = planes(w.a, m, m), p = planes(w.p, m, m);
    split_kernel<T><<<dim3(n / 64, m / 64, nb), 256, 0, stream>>>(in, parts, nparts, x[0], xt[0], range.x, k0, eps,
                                                                    range.grown[1], start);
    int rc = launch_status();
    const Output<f16> none{};
    for (int s = 0; s < steps && !rc; ++s) {
        const int turn = s % 2;  // of X
        const Depth depth = s == 0 && sizeof(T) == 2 ? Depth::kExact : Depth::kBoth;
        rc = product<Product::kGram>({x[turn], x[turn], n, m, m, a, a, gram, {}, {}, nullptr, 0, 0, 0, 0.0f}, none, batch,
                                     tiles.symmetric, depth, shares, stream);
        const Coefficients ks = coefficients(s);
        const int before = s == 0 ? -1 : range.grown[s], after = range.grown[s + 1];
        if (!rc)
            rc = product<Product::kPolynomial>({a, a, m, m, m, p, p, 1.0f, a, ks, start, before, after, 0, 0.0f}, none, batch,
                                               tiles.symmetric, Depth::kBoth, shares, stream);
        if (rc) break;
        Planes own = x[turn];
        if (depth == Depth::kExact) own.lo = nullptr;
        const Operands update{p, xt[turn], m, m, n, x[1 - turn], xt[1 - turn], power(-range.p), own, ks, start,
                              before, after, -range.x, scale};
        if (s + 1 < steps) rc = product<Product::kUpdate>(update, none, batch, tiles.update, depth, shares, stream);
        else rc = product<Product::kLast>(update, out, batch, tiles.update, depth, shares, stream);
    }
    return rc;
}

}  // namespace
}  // namespace trivance

using namespace trivance;

extern "C" {

int64_t trivance_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols) {
    if (batch < 0 || rows < 0 || cols < 0) return TRIVANCE_EINVAL;
    if (rows > kMaxSide || cols > kMaxSide || batch > 65535) return TRIVANCE_EUNSUPPORTED;
    if (batch == 0 || rows == 0 || cols == 0) return 0;
    return layout_of(batch, rows, cols).bytes;
}

int trivance_orthogonalize(const void* x, void* out, int64_t batch, int64_t rows, int64_t cols,
                           int64_t x_batch_stride, int64_t x_row_stride, int64_t out_batch_stride,
                           int64_t out_row_stride, const float* coefficients, int steps, double scale,
                           double eps, int dtype, void* workspace, int64_t workspace_bytes,
                           void* stream) {
    if (!is_float_type(dtype) || !coefficients || steps < 1 || !(eps >= 0.0) || !std::isfinite((float)scale))
        return TRIVANCE_EINVAL;
    const int64_t need = trivance_orthogonalize_workspace_bytes(batch, rows, cols);
    if (need < 0) return (int)need;
    if (steps > kMaxSteps) return TRIVANCE_EUNSUPPORTED;
    const Ranges range = ranges_of(coefficients, steps);
    if (!range.ok) return TRIVANCE_EUNSUPPORTED;
    if (batch == 0 || rows == 0 || cols == 0) return TRIVANCE_OK;
    if (!x || !out || !rows_fit(batch, rows, cols, x_batch_stride, x_row_stride) ||
        !rows_fit(batch, rows, cols, out_batch_stride, out_row_stride) ||
        !rows_distinct(batch, rows, cols, out_batch_stride, out_row_stride))
        return TRIVANCE_EINVAL;
    if (workspace_bytes < need || (need > 0 && !workspace)) return TRIVANCE_ESIZE;
    const Layout w = layout_of(batch, rows, cols);
    const bool tall = rows > cols;
    const int m = (int)(tall ? cols : rows), n = (int)(tall ? rows : cols);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto go = [&](auto type) {
        using T = decltype(type);
        return run<T>({static_cast<const T*>(x), x_batch_stride, tall ? 1 : x_row_stride,
                       tall ? x_row_stride : 1, m, n},
                      {static_cast<T*>(out), out_batch_stride, tall ? 1 : out_row_stride,
                       tall ? out_row_stride : 1, m, n},
                      batch, steps, coefficients, range, (float)scale, eps, w, workspace, s);
    };
    return dtype == TRIVANCE_F32 ? go(float{}) : dtype == TRIVANCE_BF16 ? go(bf16{}) : go(f16{});
}

}  // extern "C"
