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
// What bounds it: the MFMA rate, for matrices of some hundred rows and more.
// Layout. X is kept both ways round, so that both operands of every product have their summed index
// contiguous; sides are padded with zeros to whole tiles. A and A A are symmetric: only tiles on and
// above the diagonal are computed and each is written to both places.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "device.h"
#include "operators.h"

namespace trivance {
namespace {

constexpr float kScale = 4096.0f;  // 2^12, of every stored matrix
constexpr int kScaleExp = 12;
constexpr int kMaxSteps = 64;
constexpr int64_t kMaxSide = 1 << 16;
constexpr int kNormParts = 256;  // partial sums of a matrix's norm

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
        f16 lo;
        split(tile[q][lane], x.hi[at], lo);
        if (sizeof(T) > 2) x.lo[at] = lo;  // zero otherwise, and not read in the first step
        split(tile[lane][q], xt.hi[att], lo);
        if (sizeof(T) > 2) xt.lo[att] = lo;
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

// How a square tile of a product is computed: the rows and columns of waves that share it, and the
// values of the summed index in one stage of local memory (two stages: 64, 128 and 128 KiB). Rates
// measured with both operands in two planes, on 2048 x 8192 from 2048 and on 2048 x 2048 from
// 2048: tiles of 256 1125 and 370 TFLOP/s (64 tiles for 256 CUs), of 128 860 and 860, of 64 530 and
// 574. Larger tiles read less of the operands again; a stage of 64 halves the barriers, and tiles of 256
// have no room for it.
template <int TILE>
struct Shape;
template <>
struct Shape<256> {
    static constexpr int kRows = 2, kCols = 4, kDepth = 32;
};
template <>
struct Shape<128> {
    static constexpr int kRows = 2, kCols = 2, kDepth = 64;
};
template <>
struct Shape<64> {
    static constexpr int kRows = 2, kCols = 2, kDepth = 64;
};

// Where a stage holds 16-byte piece p of a row of DEPTH values: pieces are permuted within their row so
// that the 16 lanes that read one piece of 16 rows, and any 8 of them in order, meet different banks.
template <int DEPTH>
__device__ __forceinline__ int piece_of(int row, int p) {
    if constexpr (DEPTH == 32) return p ^ ((row >> 1 & 3) ^ (row >> 3 & 1));
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
    Planes a;        // of the polynomial
    Coefficients k;
    const Coefficients* first;  // in place of k, for each matrix
};

// C = L R'. LP and RP: the planes that are not zero. While the waves multiply one stage of the
// operands the next one is on its way into the other half of local memory, so a stage has one barrier.
template <Product KIND, int TILE, int LP, int RP, typename T>
__global__ __launch_bounds__(Shape<TILE>::kRows * Shape<TILE>::kCols * 64, TILE == 64 ? 2 : 1) void product_kernel(
    Operands o, Output<T> out) {
    using S = Shape<TILE>;
    constexpr bool kSymmetric = KIND == Product::kGram || KIND == Product::kPolynomial;
    constexpr int kThreads = S::kRows * S::kCols * 64, kDepth = S::kDepth, kPieces = kDepth / 8;
    constexpr int WM = TILE / S::kRows, WN = TILE / S::kCols, MI = WM / 16, NI = WN / 16;
    constexpr int kPlane = TILE * kPieces, kStage = (LP + RP) * kPlane;
    extern __shared__ half8 stages[];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    // one XCD's workgroups take neighbouring tiles: all rows of some columns
    const int tiles = kSymmetric ? o.rows * (o.rows + 1) / 2 : o.rows * o.cols;
    const int all = xcd_contiguous(blockIdx.x, gridDim.x);
    const int64_t b = all / tiles;
    const int tile = all % tiles;
    int ti, tj;
    if constexpr (kSymmetric) {  // ti <= tj
        tj = (int)((sqrtf(8.0f * tile + 1.0f) - 1.0f) * 0.5f);
        while ((tj + 1) * (tj + 2) / 2 <= tile) ++tj;
        while (tj * (tj + 1) / 2 > tile) --tj;
        ti = tile - tj * (tj + 1) / 2;
    } else {
        ti = tile % o.rows;
        tj = tile / o.rows;
    }
    const int i0 = ti * TILE, j0 = tj * TILE;
    const int wi = wave / S::kCols * WM, wj = wave % S::kCols * WN;
    const f16* lsrc[2] = {o.l.hi + b * o.l.batch + (int64_t)i0 * o.l.ld,
                          o.l.lo + b * o.l.batch + (int64_t)i0 * o.l.ld};
    const f16* rsrc[2] = {o.r.hi + b * o.r.batch + (int64_t)j0 * o.r.ld,
                          o.r.lo + b * o.r.batch + (int64_t)j0 * o.r.ld};
    const auto load = [&](int d, half8* stage) {
#pragma unroll
        for (int p = 0; p < LP + RP; ++p) {
            const bool left = p < LP;
            const f16* src = left ? lsrc[p] : rsrc[p - LP];
            const int64_t ld = left ? o.l.ld : o.r.ld;
#pragma unroll
            for (int q0 = 0; q0 < kPlane; q0 += kThreads) {
                const int q = q0 + threadIdx.x, row = q / kPieces;
                copy_to_local(src + row * ld + d + piece_of<kDepth>(row, q % kPieces) * 8,
                              stage + p * kPlane + q0 + wave * 64);
            }
        }
    };
    float4v acc[MI][NI] = {};
    load(0, stages);
    for (int d = 0, turn = 0; d < o.depth; d += kDepth, turn ^= 1) {
        // this stage has arrived, and every wave has read the other half
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (d + kDepth < o.depth) load(d + kDepth, stages + (turn ^ 1) * kStage);
        const half8* stage = stages + turn * kStage;
#pragma unroll
        for (int kk = 0; kk < kPieces / 4; ++kk) {
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
                            acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[pr][y], l[pl][x],
                                                                               acc[x][y], 0, 0, 0);
        }
    }
    Coefficients k = o.k;
    if (KIND == Product::kPolynomial && o.first) k = o.first[b];
#pragma unroll
    for (int x = 0; x < MI; ++x)
#pragma unroll
        for (int y = 0; y < NI; ++y) {
            const int i = i0 + wi + x * 16 + lane % 16, j = j0 + wj + y * 16 + lane / 16 * 4;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = acc[x][y][q] * (1.0f / kScale);
            if constexpr (KIND == Product::kPolynomial) {
                const int64_t at = b * o.a.batch + (int64_t)i * o.a.ld + j;
                const half4 h = *reinterpret_cast<const half4*>(o.a.hi + at);
                const half4 w = *reinterpret_cast<const half4*>(o.a.lo + at);
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
                const int64_t at = b * o.c.batch + (int64_t)i * o.c.ld + j;
                *reinterpret_cast<half4*>(o.c.hi + at) = h;
                *reinterpret_cast<half4*>(o.c.lo + at) = w;
                if (!kSymmetric || ti != tj) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int64_t att = b * o.ct.batch + (int64_t)(j + q) * o.ct.ld + i;
                        o.ct.hi[att] = h[q];
                        o.ct.lo[att] = w[q];
                    }
                }
            }
        }
}

// The tiles of a call: of the symmetric products and of the others. Sides are padded to the larger.
struct Tiles {
    int symmetric, update;
    int pad() const { return symmetric > update ? symmetric : update; }
};

int64_t padded(int64_t side, int tile) { return (side + tile - 1) / tile * tile; }

// The pair that takes the least time by the measured rates, counting whole rounds of the 256 CUs and the
// padding.
Tiles tiles_of(int64_t batch, int64_t m, int64_t n) {
    const auto cost = [&](int tile, int64_t tiles, int64_t depth) {
        const double rate = tile == 256 ? 1.0 : tile == 128 ? 0.76 : 0.5;
        return (double)((batch * tiles + 255) / 256) * tile * tile * depth / rate;
    };
    Tiles best{64, 64};
    double least = INFINITY;
    for (const int s : {64, 128})
        for (const int u : {64, 128, 256}) {
            const Tiles t{s, u};
            const int64_t pm = padded(m, t.pad()), pn = padded(n, t.pad());
            const int64_t ms = pm / s;
            const double c = cost(s, ms * (ms + 1) / 2, pn + pm) + cost(u, pm / u * (pn / u), pm);
            if (c < least) {
                least = c;
                best = t;
            }
        }
    return best;
}

// The workspace: norm parts and first coefficients, then the planes of X and X' twice, A and P.
struct Layout {
    int64_t parts, first, x[2], xt[2], a, p, bytes;  // byte offsets
    Tiles tiles;
    int m, n;
};

Layout layout_of(int64_t batch, int64_t rows, int64_t cols) {
    Layout w;
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    w.tiles = tiles_of(batch, m, n);
    w.m = (int)padded(m, w.tiles.pad());
    w.n = (int)padded(n, w.tiles.pad());
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

template <Product KIND, int TILE, int LP, int RP, typename T>
int launch_product(const Operands& o, const Output<T>& out, int64_t batch, hipStream_t stream) {
    using S = Shape<TILE>;
    constexpr bool kSymmetric = KIND == Product::kGram || KIND == Product::kPolynomial;
    constexpr size_t local = (size_t)2 * (LP + RP) * TILE * S::kDepth * sizeof(f16);
    const auto kernel = product_kernel<KIND, TILE, LP, RP, T>;
    if (local > 65536 &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)local) != hipSuccess)
        return TRIVANCE_EHIP;
    const int64_t tiles = kSymmetric ? (int64_t)o.rows * (o.rows + 1) / 2 : (int64_t)o.rows * o.cols;
    kernel<<<(unsigned)(tiles * batch), S::kRows * S::kCols * 64, local, stream>>>(o, out);
    return launch_status();
}

// A product by the call's tiles. `exact`: X0 has one plane.
template <Product KIND, typename T>
int product(Operands o, const Output<T>& out, int64_t batch, int tile, bool exact, hipStream_t stream) {
    o.rows = o.rows / tile;
    o.cols = o.cols / tile;
    // in a first step from 16 bits the lower plane of X is zero: both operands of the Gram matrix, the
    // right one of the update
    constexpr int LP = KIND == Product::kGram ? 1 : 2;
#define LAUNCH(TILE)                                                                                 \
    if (tile == TILE) {                                                                              \
        if constexpr (KIND != Product::kPolynomial)                                                  \
            if (exact) return launch_product<KIND, TILE, LP, 1>(o, out, batch, stream);              \
        return launch_product<KIND, TILE, 2, 2>(o, out, batch, stream);                              \
    }
    if constexpr (KIND == Product::kUpdate || KIND == Product::kLast) LAUNCH(256)
    LAUNCH(128)
    LAUNCH(64)
#undef LAUNCH
    return TRIVANCE_EINVAL;
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
    int rc = launch_status();
    for (int s = 0; s < steps && !rc; ++s) {
        const Coefficients c{k[3 * s], k[3 * s + 1], k[3 * s + 2]};
        const int q = s % 2;
        const bool exact = s == 0 && sizeof(T) == 2;
        const Output<f16> none{};
        rc = product<Product::kGram>({x[q], x[q], w.n, w.m, w.m, a, a, a, c, nullptr}, none, batch,
                                     w.tiles.symmetric, exact, stream);
        if (rc) break;
        rc = product<Product::kPolynomial>({a, a, w.m, w.m, w.m, p, p, a, c, s == 0 ? first : nullptr}, none,
                                           batch, w.tiles.symmetric, false, stream);
        if (rc) break;
        const Operands update{p, xt[q], w.m, w.m, w.n, x[1 - q], xt[1 - q], a, c, nullptr};
        rc = s + 1 < steps ? product<Product::kUpdate>(update, none, batch, w.tiles.update, exact, stream)
                           : product<Product::kLast>(update, out, batch, w.tiles.update, exact, stream);
    }
    return rc;
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
