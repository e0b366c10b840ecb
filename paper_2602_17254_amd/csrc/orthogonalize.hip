// Orthogonalises matrices by Newton-Schulz products: X0 = G / (|G|_F + eps), and per step
//
//   A = X X'     P = a I + b A + c A A     X <- P X
//
// on the smaller side of G (X = G' where G is taller than wide), so that every singular value s of X0
// passes the odd polynomial a s + b s^3 + c s^5 of each step and the singular vectors stay.
//
// Precision. A weak direction of G grows by up to a in every step (by 485 in five steps with
// a = 3.4445), and so does any rounding noise that falls into it: with bf16 operands five steps end 1
// to 30% off, with fp16 0.1 to 3%, by the spectrum. Every matrix is kept as two fp16 numbers hi + lo of
// 22 bits together, and a product is three MFMA products hi hi + hi lo + lo hi in fp32 sums: fp32
// accuracy for every spectrum at a third of the fp16 rate, five times the rate of fp32 MFMA. Values are
// held times 2^12: all entries are at most 15 (checked for the coefficients) and the spacing of lo
// is 2^-36. G enters scaled by a power of two, exactly where it has 16 bits; the rest of the norm goes into
// the first step's coefficients.
//
// Layout. X is kept both ways round, so that both operands of every product have their summed index
// contiguous; sides are padded with zeros to whole tiles. A and A A are symmetric: only tiles on and
// above the diagonal are computed and each is written to both places.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "operators.h"

namespace trivance {
namespace {

constexpr float kScale = 4096.0f;  // 2^12, of every stored matrix
constexpr int kScaleExp = 12;
constexpr int kMaxSteps = 64;
constexpr int64_t kMaxSide = 1 << 16;
constexpr int kNormParts = 256;  // partial sums of a matrix's norm
constexpr int kTile = 64;
constexpr int kDepth = 32;  // of one stage of a product

typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef f16 half4 __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

// A matrix in two planes, rows `ld` apart.
struct Planes {
    f16 *hi, *lo;
    int64_t batch;  // elements from one matrix to the next
    int ld;
};

struct Coefficients {
    float a, b, c;
};

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
// memory: its contiguous index runs over the lanes.
template <typename T>
__global__ __launch_bounds__(256) void norm_parts_kernel(Input<T> in, double* parts) {
    __shared__ double sums[4];
    const bool tall = in.sj != 1;
    const int rows = tall ? in.n : in.m, cols = tall ? in.m : in.n;
    const int64_t stride = tall ? in.sj : in.si;
    const T* x = in.x + blockIdx.y * in.batch;
    double s = 0.0;
    for (int i = blockIdx.x; i < rows; i += gridDim.x)
        for (int j = threadIdx.x; j < cols; j += 256) {
            const double v = (float)x[i * stride + j];
            s += v * v;
        }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        parts[blockIdx.y * kNormParts + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// X both ways round, scaled by 2^12 over the power of two below the norm and padded with zeros, and the
// first step's coefficients, which hold what is left of the norm.
template <typename T>
__global__ __launch_bounds__(256) void split_kernel(Input<T> in, const double* parts, int nparts,
                                                    Planes x, Planes xt, Coefficients c, float eps,
                                                    Coefficients* first) {
    __shared__ float tile[64][65];
    const int64_t b = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x % 64; i < nparts; i += 64) sum += parts[b * kNormParts + i];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    const double norm = sqrt(sum);
    int e = 0;
    if (norm > 0.0 && norm < __builtin_inf()) e = ilogb(norm);
    // zero for a zero matrix; not a number where the norm is none
    const double alpha = norm == 0.0 ? 0.0 : (norm < __builtin_inf() ? ldexp(1.0, e) / (norm + eps) : __builtin_nan(""));
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    if (i0 == 0 && j0 == 0 && threadIdx.x == 0)
        first[b] = {(float)(c.a * alpha), (float)(c.b * (alpha * alpha * alpha)),
                    (float)(c.c * (alpha * alpha * alpha * alpha * alpha))};
    const T* g = in.x + b * in.batch;
    const bool tall = in.sj != 1;
    const int lane = threadIdx.x % 64;
    for (int q = threadIdx.x / 64; q < 64; q += 4) {
        const int i = tall ? i0 + lane : i0 + q, j = tall ? j0 + q : j0 + lane;
        const float v = i < in.m && j < in.n ? (float)g[i * in.si + j * in.sj] : 0.0f;
        if (tall) tile[lane][q] = ldexpf(v, kScaleExp - e);
        else tile[q][lane] = ldexpf(v, kScaleExp - e);
    }
    __syncthreads();
    for (int q = threadIdx.x / 64; q < 64; q += 4) {
        const int64_t at = b * x.batch + (int64_t)(i0 + q) * x.ld + j0 + lane;
        const int64_t att = b * xt.batch + (int64_t)(j0 + q) * xt.ld + i0 + lane;
        split(tile[q][lane], x.hi[at], x.lo[at]);
        split(tile[lane][q], xt.hi[att], xt.lo[att]);
    }
}

enum class Product { kGram, kPolynomial, kUpdate, kLast };

template <typename T>
struct Output {
    T* x;
    int64_t batch, si, sj;
    int m, n;
    float scale;
};

// One stage of an operand: kTile rows of kDepth values in 16-byte pieces. The piece of row r and
// index p lies at piece p ^ (r / 4 % 4), so that 16 rows' pieces of one index fall into 16
// different groups of banks.
__device__ __forceinline__ int piece(int row, int p) { return row * (kDepth / 8) + (p ^ (row / 4 % 4)); }

// C = L R' over `depth` (whole stages): L's rows are C's rows and R's rows C's columns. One workgroup of
// four waves a tile, each wave a quarter.
template <Product KIND, typename T>
__global__ __launch_bounds__(256) void product_kernel(Planes l, Planes r, int depth, Planes c, Planes ct,
                                                      Planes a, Coefficients k,
                                                      const Coefficients* first, Output<T> out) {
    constexpr bool kSymmetric = KIND == Product::kGram || KIND == Product::kPolynomial;
    if (kSymmetric && blockIdx.x < blockIdx.y) return;
    __shared__ half8 stage[4][kTile * kDepth / 8];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t b = blockIdx.z;
    const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;
    const f16* src[4] = {l.hi + b * l.batch + (int64_t)i0 * l.ld, l.lo + b * l.batch + (int64_t)i0 * l.ld,
                         r.hi + b * r.batch + (int64_t)j0 * r.ld, r.lo + b * r.batch + (int64_t)j0 * r.ld};
    const int wi = wave / 2 * 32, wj = wave % 2 * 32;
    float4v acc[2][2] = {};
    const int row = threadIdx.x / 4, p = threadIdx.x % 4;
    for (int d = 0; d < depth; d += kDepth) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q)
            stage[q][piece(row, p)] =
                *reinterpret_cast<const half8*>(src[q] + (int64_t)row * (q < 2 ? l.ld : r.ld) + d + p * 8);
        __syncthreads();
        half8 f[4][2];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int s = 0; s < 2; ++s)
                f[q][s] = stage[q][piece((q < 2 ? wi : wj) + s * 16 + lane % 16, lane / 16)];
        // R first: a lane then holds four consecutive columns of one row
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[3][y], f[0][x], acc[x][y], 0, 0, 0);
                acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[2][y], f[1][x], acc[x][y], 0, 0, 0);
                acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[2][y], f[0][x], acc[x][y], 0, 0, 0);
            }
    }
    if (KIND == Product::kPolynomial && first) k = first[b];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int i = i0 + wi + x * 16 + lane % 16, j = j0 + wj + y * 16 + lane / 16 * 4;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = acc[x][y][q] * (1.0f / kScale);
            if constexpr (KIND == Product::kPolynomial) {
                const int64_t at = b * a.batch + (int64_t)i * a.ld + j;
                const half4 h = *reinterpret_cast<const half4*>(a.hi + at);
                const half4 w = *reinterpret_cast<const half4*>(a.lo + at);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    v[q] = k.b * ((float)h[q] + (float)w[q]) + k.c * v[q] + (i == j + q ? k.a * kScale : 0.0f);
            }
            if constexpr (KIND == Product::kLast) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (i < out.m && j + q < out.n)
                        out.x[b * out.batch + i * out.si + (j + q) * out.sj] =
                            (T)(v[q] * (out.scale / kScale));
            } else {
                half4 h, w;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f16 hi, lo;
                    split(v[q], hi, lo);
                    h[q] = hi;
                    w[q] = lo;
                }
                const int64_t at = b * c.batch + (int64_t)i * c.ld + j;
                *reinterpret_cast<half4*>(c.hi + at) = h;
                *reinterpret_cast<half4*>(c.lo + at) = w;
                if (!kSymmetric || blockIdx.x != blockIdx.y) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int64_t att = b * ct.batch + (int64_t)(j + q) * ct.ld + i;
                        ct.hi[att] = h[q];
                        ct.lo[att] = w[q];
                    }
                }
            }
        }
}

int pad(int64_t side) { return (int)((side + kTile - 1) / kTile * kTile); }

// The workspace: norm parts and first coefficients, then the planes of X and X' twice, A and P.
struct Layout {
    int64_t parts, first, x[2], xt[2], a, p, bytes;  // byte offsets
    int m, n;
};

Layout layout_of(int64_t batch, int64_t rows, int64_t cols) {
    Layout w;
    w.m = pad(rows < cols ? rows : cols);
    w.n = pad(rows < cols ? cols : rows);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const int64_t xs = batch * w.m * w.n * 2 * (int64_t)sizeof(f16);
    const int64_t as = batch * w.m * w.m * 2 * (int64_t)sizeof(f16);
    w.parts = take(batch * kNormParts * (int64_t)sizeof(double));
    w.first = take(batch * (int64_t)sizeof(Coefficients));
    for (int i = 0; i < 2; ++i) {
        w.x[i] = take(xs);
        w.xt[i] = take(xs);
    }
    w.a = take(as);
    w.p = take(as);
    w.bytes = at + 256;
    return w;
}

template <typename T>
int run(Input<T> in, Output<T> out, int64_t batch, int steps, const float* k, float eps, const Layout& w,
        void* workspace, hipStream_t stream) {
    char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) / 256 * 256);
    const auto planes = [&](int64_t offset, int rows, int ld) {
        f16* hi = reinterpret_cast<f16*>(base + offset);
        return Planes{hi, hi + batch * rows * ld, (int64_t)rows * ld, ld};
    };
    double* parts = reinterpret_cast<double*>(base + w.parts);
    Coefficients* first = reinterpret_cast<Coefficients*>(base + w.first);
    Planes x[2], xt[2];
    for (int i = 0; i < 2; ++i) {
        x[i] = planes(w.x[i], w.m, w.n);
        xt[i] = planes(w.xt[i], w.n, w.m);
    }
    const Planes a = planes(w.a, w.m, w.m), p = planes(w.p, w.m, w.m);
    const int rows = in.sj != 1 ? in.n : in.m;
    const int nparts = rows < kNormParts ? rows : kNormParts;
    const unsigned nb = (unsigned)batch;
    norm_parts_kernel<T><<<dim3(nparts, nb), 256, 0, stream>>>(in, parts);
    split_kernel<T><<<dim3(w.n / 64, w.m / 64, nb), 256, 0, stream>>>(
        in, parts, nparts, x[0], xt[0], Coefficients{k[0], k[1], k[2]}, eps, first);
    const dim3 square(w.m / kTile, w.m / kTile, nb), wide(w.n / kTile, w.m / kTile, nb);
    for (int s = 0; s < steps; ++s) {
        const Coefficients c{k[3 * s], k[3 * s + 1], k[3 * s + 2]};
        const int q = s % 2;
        product_kernel<Product::kGram, T><<<square, 256, 0, stream>>>(x[q], x[q], w.n, a, a, a, c, nullptr, out);
        product_kernel<Product::kPolynomial, T><<<square, 256, 0, stream>>>(
            a, a, w.m, p, p, a, c, s == 0 ? first : nullptr, out);
        if (s + 1 < steps)
            product_kernel<Product::kUpdate, T><<<wide, 256, 0, stream>>>(p, xt[q], w.m, x[1 - q], xt[1 - q],
                                                                          a, c, nullptr, out);
        else
            product_kernel<Product::kLast, T><<<wide, 256, 0, stream>>>(p, xt[q], w.m, x[q], xt[q], a, c,
                                                                        nullptr, out);
    }
    return launch_status();
}

// Whether the stored numbers stay in fp16's range for every singular value in [0, 1]: step by step, the
// largest singular value stays below 3.9 and P's within 15.
bool coefficients_ok(const float* k, int steps) {
    double most = 1.0;  // the largest singular value so far
    for (int s = 0; s < steps; ++s) {
        const double a = k[3 * s], b = k[3 * s + 1], c = k[3 * s + 2];
        double next = 0.0;
        constexpr int kSamples = 4096;
        for (int i = 0; i <= kSamples; ++i) {
            const double v = most * i / kSamples, p = a + v * v * (b + v * v * c);
            if (!(std::fabs(p) <= 15.0)) return false;
            if (std::fabs(p * v) > next) next = std::fabs(p * v);
        }
        most = next * 1.001;  // between the samples, and the rounding of the products
        if (!(most <= 3.9)) return false;
    }
    return true;
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
    if (!is_float_type(dtype) || !coefficients || steps < 1 || !(eps >= 0.0) || !std::isfinite(scale))
        return TRIVANCE_EINVAL;
    const int64_t need = trivance_orthogonalize_workspace_bytes(batch, rows, cols);
    if (need < 0) return (int)need;
    if (steps > kMaxSteps || !coefficients_ok(coefficients, steps)) return TRIVANCE_EUNSUPPORTED;
    if (need == 0) return TRIVANCE_OK;
    if (!x || !out || !rows_fit(batch, rows, cols, x_batch_stride, x_row_stride) ||
        !rows_fit(batch, rows, cols, out_batch_stride, out_row_stride) ||
        !rows_distinct(batch, rows, cols, out_batch_stride, out_row_stride))
        return TRIVANCE_EINVAL;
    if (workspace_bytes < need || !workspace) return TRIVANCE_ESIZE;
    const Layout w = layout_of(batch, rows, cols);
    const bool tall = rows > cols;
    const int m = (int)(tall ? cols : rows), n = (int)(tall ? rows : cols);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const auto go = [&](auto type) {
        using T = decltype(type);
        return run<T>({static_cast<const T*>(x), x_batch_stride, tall ? 1 : x_row_stride,
                       tall ? x_row_stride : 1, m, n},
                      {static_cast<T*>(out), out_batch_stride, tall ? 1 : out_row_stride,
                       tall ? out_row_stride : 1, m, n, (float)scale},
                      batch, steps, coefficients, (float)eps, w, workspace, s);
    };
    return dtype == TRIVANCE_F32 ? go(float{}) : dtype == TRIVANCE_BF16 ? go(bf16{}) : go(f16{});
}

}  // extern "C"
