// Orthogonalising an update by Newton-Schulz products (oz_orthogonalise): X = G / (|G|_F + eps), then a number of times
//     S = X X^T,   P = b S + c S S,   X <- a X + P X
// on the shorter side of G, which drives the singular values of X towards a common value and leaves its singular vectors.
//
// The products run on the 16-bit tensor pipe to the accuracy of FP32.  An iterate held in 16 bits would not do: what is lost in a step
// is taken up by up to |a| (3.44 with the usual coefficients) in each of the next, and the update is off by 2e-3 beyond its own
// rounding.  So a matrix is the sum of two half-precision planes hi + lo, 22 bits, of its elements times a power of two that
// uses the range up to 2^15: hi is the rounded element, lo the rounded rest.  Of the four plane products lo lo lies below the last bit; the
// other three go into one accumulator (PLANES = 2 of the product core).  Elements above 2^-18 of the bound keep all 22 bits, smaller ones an
// absolute 2^-40 of it.
//
// Planes in memory: [matrix][line][chunk of 64 elements][hi, lo][64], so that both halves of an element lie at a fixed distance, and a block
// of an operand is the same box whether its lines or its elements are the inner dimension.  Elements behind the last are zero.
//
// S and P are symmetric: only tiles on and below the diagonal are computed, those below are stored twice.  (Tiles on it are stored
// as computed.)  X keeps its r rows consecutive: for X X^T it is an operand stored along its rows, for P X one stored along the inner dimension,
// both by the same bulk copies, and S and P are read along whichever direction suits.
//
// Launches: sum of squares, planes of X, then three products a step.  Floor: (r r c + r r r + 2 r r c) operations a step and matrix,
// three times that on the pipe.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <cmath>
#include <type_traits>

#include "oz_product16.cuh"

namespace oz {
namespace {

constexpr int kMaxSteps = 100;
constexpr int NORM_THREADS = 256;
constexpr int MAX_PARTS = 64;                      // partial sums of squares of a matrix
constexpr int PLANE_TILE = 64;

__device__ __forceinline__ float load_number(const void *X, int64_t at, int type)
{
    if (type == OZ_F32) return static_cast<const float *>(X)[at];
    if (type == OZ_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(X)[at]);
    return __half2float(static_cast<const __half *>(X)[at]);
}

template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_float(float v) { return v; }

__device__ __forceinline__ void store_number(void *X, int64_t at, float v, int type)
{
    if (type == OZ_F32) static_cast<float *>(X)[at] = v;
    else if (type == OZ_BF16) static_cast<__nv_bfloat16 *>(X)[at] = __float2bfloat16_rn(v);
    else static_cast<__half *>(X)[at] = __float2half_rn(v);
}

// v as the sum of two half-precision numbers: the difference is exact, the second rounding is off by 2^-22 of v at most
__device__ __forceinline__ void split_planes(float v, __half *hi, __half *lo)
{
    *hi = __float2half_rn(v);
    *lo = __float2half_rn(v - __half2float(*hi));
}

struct MatrixParams {
    int64_t m, n, count, ldg, strideG, ldo, strideO;
    const void *G;
    void *O;
    int type, otype;
    int transposed;                 // m > n: X is the transpose of G
    int r, c, ld;                   // X is r x c, r <= c, its columns ld half-precision numbers apart
    int parts;
    double *sums;                   // [count][parts]
    double eps;
    float scale;                    // of the planes
    __half *X;                      // plane pairs: [count][c][ld]
    unsigned int *status;
};

// where element i of a line of plane pairs lies; its lo half is 64 numbers on
__device__ __forceinline__ int pair_at(int i) { return (i >> 6) * 128 + (i & 63); }

// Sums of squares, in double: any finite FP32 number squares without overflow, and the order is fixed.
__global__ void __launch_bounds__(NORM_THREADS) norm_kernel(const MatrixParams p)
{
    __shared__ double warp_sums[NORM_THREADS / 32];
    dependency_release();
    dependency_wait();
    const int64_t matrix = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts;
    const int64_t total = p.m * p.n;
    double sum = 0.0;
    for (int64_t e = part * NORM_THREADS + threadIdx.x; e < total; e += p.parts * NORM_THREADS) {
        const int64_t j = total <= 0xFFFFFFFFll ? static_cast<uint32_t>(e) / static_cast<uint32_t>(p.m) : e / p.m;
        const double v = load_number(p.G, matrix * p.strideG + (e - j * p.m) + j * p.ldg, p.type);
        sum = fma(v, v, sum);
    }
    for (int d = 16; d > 0; d /= 2) sum += __shfl_down_sync(0xFFFFFFFFu, sum, d);
    if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NORM_THREADS / 32; ++w) sum += warp_sums[w];
        p.sums[blockIdx.x] = sum;
    }
}

// 1 / (|G|_F + eps); 0 for a matrix of zeros; NaN, which the whole update then is, for one that holds Inf or NaN.  One warp.
__device__ double inverse_norm(const MatrixParams &p, int64_t matrix)
{
    double sum = 0.0;
    for (int i = threadIdx.x % 32; i < p.parts; i += 32) sum += p.sums[matrix * p.parts + i];
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (!(sum <= 1.7e308)) {
        atomicOr(p.status, 1u << OZ_ERR_NONFINITE_INPUT);
        return nan("");
    }
    return sum > 0.0 ? 1.0 / (sqrt(sum) + p.eps) : 0.0;
}

// Planes of X, tiles of 64 x 64 through shared memory where X is the transpose of G.  PLANES = false: no step follows, X itself
// goes to O, in G's own direction.
template <bool PLANES>
__global__ void __launch_bounds__(256) planes_kernel(const MatrixParams p)
{
    __shared__ float tile[PLANE_TILE][PLANE_TILE + 1];
    __shared__ double factor;
    dependency_release();
    dependency_wait();
    const int64_t rows = p.m, cols = p.n;
    const int64_t tiles_m = (rows + PLANE_TILE - 1) / PLANE_TILE, each = tiles_m * ((cols + PLANE_TILE - 1) / PLANE_TILE);
    const int64_t matrix = blockIdx.x / each, t = blockIdx.x % each;
    const int64_t i0 = t % tiles_m * PLANE_TILE, j0 = t / tiles_m * PLANE_TILE;
    if (threadIdx.x < 32) {
        const double f = inverse_norm(p, matrix);
        if (threadIdx.x == 0) factor = f;
    }
    __syncthreads();
    const double f = PLANES ? factor * static_cast<double>(p.scale) : factor;
    const int ti = threadIdx.x % PLANE_TILE, tj = threadIdx.x / PLANE_TILE;
#pragma unroll
    for (int s = 0; s < PLANE_TILE; s += 4) {
        const int64_t i = i0 + ti, j = j0 + tj + s;
        float v = 0.0f;
        if (i < rows && j < cols) {
            v = static_cast<float>(static_cast<double>(load_number(p.G, matrix * p.strideG + i + j * p.ldg, p.type)) * f);
            if (!PLANES) store_number(p.O, matrix * p.strideO + i + j * p.ldo, v, p.otype);
        }
        if (PLANES) tile[tj + s][ti] = v;
    }
    if (!PLANES) return;
    __syncthreads();
    const int64_t x0 = p.transposed ? j0 : i0, y0 = p.transposed ? i0 : j0;       // first row and column of X
#pragma unroll
    for (int s = 0; s < PLANE_TILE; s += 4) {
        // rows behind the last are written too: the tile holds zeros there
        const int64_t x = x0 + ti, y = y0 + tj + s;
        const float v = p.transposed ? tile[ti][tj + s] : tile[tj + s][ti];
        if (y < p.c) {
            __half *to = p.X + (matrix * p.c + y) * p.ld + pair_at(static_cast<int>(x));
            split_planes(v, to, to + 64);
        }
    }
}

// ---------------------------------------------------------------- products
enum { kGram, kPolynomial, kApply, kApplyLast };

struct NewtonParams {
    int count, r, c, ld;
    float alpha, beta;              // result = alpha accumulator + beta old
    const __half *old;              // plane pairs [count][r or c][ld]: S of kPolynomial, X of kApply
    __half *out;                    // plane pairs
    void *O;                        // kApplyLast
    int64_t ldo, strideO;
    int otype, transposed;
    Core16 core;
};

template <int MODE>
struct NewtonPolicy {
    using Params = NewtonParams;
    struct Tile : Tile16 {
        int matrix, j0;
        bool mirror;
    };
    static constexpr bool RAGGED_K = false, SYMMETRIC = MODE == kGram || MODE == kPolynomial;

    static __device__ __forceinline__ void setup(const Params &, int, int *) {}

    template <int CG, int BN>
    static __device__ __forceinline__ uint32_t tiles_each(const Params &p)
    {
        const uint32_t tm = static_cast<uint32_t>((p.r + 128 * CG - 1) / (128 * CG));
        static_assert(!SYMMETRIC || 128 * CG == BN, "square tiles");
        return SYMMETRIC ? tm * (tm + 1) / 2 : tm * static_cast<uint32_t>((p.c + BN - 1) / BN);
    }

    template <int CG, int BN>
    static __device__ __forceinline__ int64_t total(const Params &p, const int *)
    {
        return static_cast<int64_t>(p.count) * tiles_each<CG, BN>(p);
    }

    template <int CG, int BN>
    static __device__ __forceinline__ Tile decode(const Params &p, const int *, int64_t item)
    {
        const uint32_t each = tiles_each<CG, BN>(p);
        Tile t;
        t.matrix = static_cast<int>(static_cast<uint32_t>(item) / each);
        const uint32_t in = static_cast<uint32_t>(item) - static_cast<uint32_t>(t.matrix) * each;
        uint32_t ti, tj;
        if (SYMMETRIC) {
            ti = static_cast<uint32_t>((sqrtf(8.0f * static_cast<float>(in) + 1.0f) - 1.0f) * 0.5f);
            while (ti * (ti + 1) / 2 > in) --ti;
            while ((ti + 1) * (ti + 2) / 2 <= in) ++ti;
            tj = in - ti * (ti + 1) / 2;
        } else {
            const uint32_t tm = static_cast<uint32_t>((p.r + 128 * CG - 1) / (128 * CG));
            ti = in % tm;
            tj = in / tm;
        }
        t.mirror = SYMMETRIC && ti != tj;
        t.a_row = static_cast<int>(ti) * 128 * CG;
        t.b_row = t.j0 = static_cast<int>(tj) * BN;
        t.a_z = t.b_z = t.matrix;
        t.k_begin = 0;
        t.k_len = MODE == kGram ? p.c : p.r;
        const int left = (SYMMETRIC ? p.r : p.c) - t.j0;
        // (an operand along its rows comes in whole chunks: half of the columns from each CTA)
        constexpr int GRAIN = MODE == kGram ? 64 * CG : 16 * CG;
        t.cols = left >= BN ? BN : (left + GRAIN - 1) / GRAIN * GRAIN;
        return t;
    }

    // A thread has one row of X, S or P (consecutive lanes consecutive rows) and N columns, eight at a time at most.
    template <int CG, int BN, int N>
    static __device__ __forceinline__ void store(const Params &p, const Tile &t, const float (&acc)[N], int row, int col)
    {
        const int i = t.a_row + row, j0 = t.j0 + col, lines = SYMMETRIC ? p.r : p.c, left = lines - j0;
        if (i >= (MODE == kApplyLast ? p.r : p.ld / 2) || left <= 0) return;
        if (left >= N) store_columns<true>(p, t, acc, i, j0, lines, left);
        else store_columns<false>(p, t, acc, i, j0, lines, left);
    }

    template <bool FULL, int N>
    static __device__ __forceinline__ void store_columns(const Params &p, const Tile &t, const float (&acc)[N], int i, int j0, int lines, int left)
    {
        constexpr int STEP = N < 8 ? N : 8;
        const int64_t base = static_cast<int64_t>(t.matrix) * lines * p.ld, at = base + static_cast<int64_t>(j0) * p.ld + pair_at(i);
        const __half *old = MODE == kGram ? nullptr : p.old + at;
        // some results: alpha accumulator + beta old
        auto results = [&](float (&v)[STEP], int c0) {
            __half hi[STEP], lo[STEP];
            if constexpr (MODE != kGram) {
#pragma unroll
                for (int c = 0; c < STEP; ++c) {
                    const bool inside = FULL || c0 + c < left;
                    hi[c] = inside ? old[0] : __half();
                    lo[c] = inside ? old[64] : __half();
                    old += p.ld;
                }
            }
#pragma unroll
            for (int c = 0; c < STEP; ++c) {
                v[c] = p.alpha * acc[c0 + c];
                if constexpr (MODE != kGram) v[c] = fmaf(p.beta, __half2float(hi[c]) + __half2float(lo[c]), v[c]);
            }
        };
        if constexpr (MODE == kApplyLast) {
            auto as = [&](auto *O) {
                using T = typename std::remove_pointer<decltype(O)>::type;
                O += t.matrix * p.strideO;
                if (p.transposed) {
                    // the row's elements are consecutive
                    constexpr int WIDE = STEP * static_cast<int>(sizeof(T)) / 16;
                    T *to = O + j0 + i * p.ldo;
                    const bool wide = FULL && reinterpret_cast<uintptr_t>(to) % 16 == 0;
#pragma unroll
                    for (int c0 = 0; c0 < N; c0 += STEP) {
                        float v[STEP];
                        results(v, c0);
                        __align__(16) T w[STEP];
#pragma unroll
                        for (int c = 0; c < STEP; ++c) w[c] = from_float<T>(v[c]);
                        if (WIDE > 0 && wide) {
#pragma unroll
                            for (int c = 0; c < WIDE; ++c) reinterpret_cast<uint4 *>(to + c0)[c] = reinterpret_cast<const uint4 *>(w)[c];
                        } else {
#pragma unroll
                            for (int c = 0; c < STEP; ++c)
                                if (FULL || c0 + c < left) to[c0 + c] = w[c];
                        }
                    }
                } else {
                    T *to = O + i + j0 * p.ldo;
#pragma unroll
                    for (int c0 = 0; c0 < N; c0 += STEP) {
                        float v[STEP];
                        results(v, c0);
#pragma unroll
                        for (int c = 0; c < STEP; ++c) {
                            if (FULL || c0 + c < left) *to = from_float<T>(v[c]);
                            to += p.ldo;
                        }
                    }
                }
            };
            if (p.otype == OZ_F32) as(static_cast<float *>(p.O));
            else if (p.otype == OZ_BF16) as(static_cast<__nv_bfloat16 *>(p.O));
            else as(static_cast<__half *>(p.O));
        } else {
            __half *to = p.out + at;
            // The same elements of the other triangle: elements j0 .. of line i, where that is one.  Behind the last column they are the zeros that
            // belong there.
            __half *mirror = p.out + base + static_cast<int64_t>(i) * p.ld + pair_at(j0);
            const bool mirrored = SYMMETRIC && t.mirror && i < lines;
#pragma unroll
            for (int c0 = 0; c0 < N; c0 += STEP) {
                float v[STEP];
                __align__(16) __half hi[STEP], lo[STEP];
                results(v, c0);
#pragma unroll
                for (int c = 0; c < STEP; ++c) split_planes(v[c], &hi[c], &lo[c]);
#pragma unroll
                for (int c = 0; c < STEP; ++c) {
                    if (FULL || c0 + c < left) {
                        to[0] = hi[c];
                        to[64] = lo[c];
                    }
                    to += p.ld;
                }
                static_assert(!SYMMETRIC || STEP == 8, "whole vectors");
                if (mirrored && (FULL || c0 < left)) {
                    *reinterpret_cast<uint4 *>(mirror + c0) = *reinterpret_cast<const uint4 *>(hi);
                    *reinterpret_cast<uint4 *>(mirror + c0 + 64) = *reinterpret_cast<const uint4 *>(lo);
                }
            }
        }
    }
};

template <int MODE>
oz_status_t launch_newton(NewtonParams &p, const CUtensorMap &mapA, const CUtensorMap &mapB, cudaStream_t stream)
{
    constexpr bool SYMMETRIC = NewtonPolicy<MODE>::SYMMETRIC;
    const int64_t tm = (p.r + 255) / 256, tiles = p.count * (SYMMETRIC ? tm * (tm + 1) / 2 : tm * ((p.c + 255) / 256));
    p.core.a_mn = p.core.b_mn = MODE == kGram;
    p.core.idesc = idesc16(false, p.core.a_mn, p.core.b_mn, 2);
    // Tiles are always 256 x 256 by pairs: the three plane products of a block read shared memory at 106 bytes a cycle; those of tiles of 128 x 128 by
    // single CTAs would at 213 of the 128 that it has.  Few tiles are shared out along the inner dimension.
    const int64_t pairs = sm_count() / 2;
    if (4 * tiles <= pairs) return launch_product16<NewtonPolicy<MODE>, 2, 256, 2, 4>(mapA, mapB, p, tiles, 0, stream);
    if (2 * tiles <= pairs) return launch_product16<NewtonPolicy<MODE>, 2, 256, 2, 2>(mapA, mapB, p, tiles, 0, stream);
    return launch_product16<NewtonPolicy<MODE>, 2, 256, 2, 1>(mapA, mapB, p, tiles, 0, stream);
}

// ---------------------------------------------------------------- host side
struct Layout {
    int64_t r, c, chunks;
    int parts;
    size_t sums, x[2], s, poly, total;
};

Layout layout_of(int64_t m, int64_t n, int64_t count)
{
    Layout l{};
    l.r = m < n ? m : n;
    l.c = m < n ? n : m;
    l.chunks = (l.r + 63) / 64;
    const int64_t pieces = (m * n + NORM_THREADS * 16 - 1) / (NORM_THREADS * 16);
    l.parts = static_cast<int>(pieces < MAX_PARTS ? pieces : MAX_PARTS);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += static_cast<size_t>(round_up(bytes, 256));
        return here;
    };
    l.sums = take(count * l.parts * 8);
    l.x[0] = take(count * l.c * l.chunks * 256);
    l.x[1] = take(count * l.c * l.chunks * 256);
    l.s = take(count * l.r * l.chunks * 256);
    l.poly = take(count * l.r * l.chunks * 256);
    l.total = at;
    return l;
}

bool valid_shape(int64_t m, int64_t n, int64_t count)
{
    // 2^40 bytes bound the elements of a matrix' planes: every index that the kernels form in 32 bits fits
    return m <= OZ_EXTENT_MAX && n <= OZ_EXTENT_MAX && count <= OZ_EXTENT_MAX && (m == 0 || n <= (1ll << 38) / m) &&
           (m * n == 0 || count <= (1ll << 38) / (m * n));
}

// the largest |a s + b s^3 + c s^5| of 0 <= s <= bound: at the end or where a + 3 b q + 5 c q^2 = 0, q = s^2
double largest_value(double a, double b, double c, double bound)
{
    auto value = [&](double q) { return std::fabs(std::sqrt(q) * (a + q * (b + q * c))); };
    double most = value(bound * bound);
    const double d = 9.0 * b * b - 20.0 * a * c;
    double roots[2] = {-1.0, -1.0};
    if (c != 0.0 && d >= 0.0) {
        roots[0] = (-3.0 * b + std::sqrt(d)) / (10.0 * c);
        roots[1] = (-3.0 * b - std::sqrt(d)) / (10.0 * c);
    } else if (c == 0.0 && b != 0.0) {
        roots[0] = -a / (3.0 * b);
    }
    for (double q : roots)
        if (q > 0.0 && q < bound * bound && value(q) > most) most = value(q);
    return most;
}

// the largest |b q + c q^2| of 0 <= q <= bound
double largest_polynomial(double b, double c, double bound)
{
    double most = std::fabs(bound * (b + bound * c));
    const double q = c != 0.0 ? -b / (2.0 * c) : -1.0;
    if (q > 0.0 && q < bound && std::fabs(q * (b + q * c)) > most) most = std::fabs(q * (b + q * c));
    return most;
}

// a power of two that takes numbers of up to `bound` (and 1 percent for the roundings on the way) to at most 2^15; 2^60 at most, so
// that quotients of three of them are FP32 numbers
double plane_scale(double bound)
{
    int e = -45;
    if (bound > 0x1p-46) std::frexp(bound * 1.01, &e);           // bound * 1.01 <= 2^e
    return std::ldexp(1.0, 15 - e);
}

}  // namespace
}  // namespace oz

using namespace oz;

extern "C" {

size_t oz_orthogonalise_workspace_bytes(int64_t m, int64_t n, int64_t count)
{
    if (m < 0 || n < 0 || count < 0 || !valid_shape(m, n, count) || m == 0 || n == 0 || count == 0) return 0;
    return layout_of(m, n, count).total;
}

oz_status_t oz_orthogonalise(int64_t m, int64_t n, int64_t count, oz_type_t type, const void *G, int64_t ldg, int64_t strideG, int steps,
                             const double *coefficients, double eps, oz_type_t otype, void *O, int64_t ldo, int64_t strideO,
                             void *workspace, size_t bytes, void *stream)
{
    if (m < 0 || n < 0 || count < 0 || steps < 0) return OZ_ERR_INVALID_ARG;
    auto valid_type = [](int t) { return t == OZ_BF16 || t == OZ_F16 || t == OZ_F32; };
    if (!valid_type(type) || !valid_type(otype)) return OZ_ERR_INVALID_ARG;
    if ((steps > 0 && !coefficients) || !(eps >= 0.0) || !std::isfinite(eps)) return OZ_ERR_INVALID_ARG;
    if (!valid_shape(m, n, count) || steps > kMaxSteps) return OZ_ERR_UNSUPPORTED;
    // the largest singular value of X before each step, and of the result
    double bound[kMaxSteps + 1] = {1.0};
    const double a = steps ? coefficients[0] : 0.0, b = steps ? coefficients[1] : 0.0, c = steps ? coefficients[2] : 0.0;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return OZ_ERR_INVALID_ARG;
    for (int s = 0; s < steps; ++s) {
        bound[s + 1] = largest_value(a, b, c, bound[s]);
        const double poly = largest_polynomial(b, c, bound[s] * bound[s]);
        if (!(bound[s + 1] <= 0x1p30) || !(poly <= 0x1p60) || (bound[s + 1] < 0x1p-30)) return OZ_ERR_UNSUPPORTED;
    }
    if (m == 0 || n == 0 || count == 0) return OZ_OK;
    const size_t in = type == OZ_F32 ? 4 : 2, out = otype == OZ_F32 ? 4 : 2;
    if (!G || !O || reinterpret_cast<uintptr_t>(G) % in || reinterpret_cast<uintptr_t>(O) % out || ldg < m || ldo < m) return OZ_ERR_INVALID_ARG;
    if (count > 1 && (strideG < 0 || strideO < m || (strideO - m) / ldo < n - 1)) return OZ_ERR_INVALID_ARG;
    const Layout l = layout_of(m, n, count);
    if (!workspace || bytes < l.total) return OZ_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return OZ_ERR_INVALID_ARG;
    oz_status_t st = ensure_device_ready();
    if (st != OZ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    __half *x[2] = {reinterpret_cast<__half *>(ws + l.x[0]), reinterpret_cast<__half *>(ws + l.x[1])};
    __half *gram = reinterpret_cast<__half *>(ws + l.s), *poly = reinterpret_cast<__half *>(ws + l.poly);
    CUtensorMap map_x[2], map_s, map_p;
    if (steps && !(make_pair_map16(&map_x[0], x[0], l.chunks, l.c, count) && make_pair_map16(&map_x[1], x[1], l.chunks, l.c, count) &&
                   make_pair_map16(&map_s, gram, l.chunks, l.r, count) && make_pair_map16(&map_p, poly, l.chunks, l.r, count)))
        return OZ_ERR_CUDA;

    MatrixParams mp{};
    mp.m = m;
    mp.n = n;
    mp.count = count;
    mp.ldg = ldg;
    mp.strideG = strideG;
    mp.ldo = ldo;
    mp.strideO = strideO;
    mp.G = G;
    mp.O = O;
    mp.type = type;
    mp.otype = otype;
    mp.transposed = m > n;
    mp.r = static_cast<int>(l.r);
    mp.c = static_cast<int>(l.c);
    mp.ld = static_cast<int>(128 * l.chunks);
    mp.parts = l.parts;
    mp.sums = reinterpret_cast<double *>(ws + l.sums);
    mp.eps = eps;
    mp.scale = static_cast<float>(plane_scale(bound[0]));
    mp.X = x[0];
    mp.status = device_status_word();
    const int64_t tiles = count * ((m + PLANE_TILE - 1) / PLANE_TILE) * ((n + PLANE_TILE - 1) / PLANE_TILE);
    if (tiles > 0x7FFFFFFF || count * l.parts > 0x7FFFFFFF) return OZ_ERR_UNSUPPORTED;
    OZ_CUDA_CHECK(launch(norm_kernel, dim3(static_cast<unsigned>(count * l.parts)), NORM_THREADS, 0, s, mp));
    OZ_CUDA_CHECK(launch(steps ? planes_kernel<true> : planes_kernel<false>, dim3(static_cast<unsigned>(tiles)), 256, 0, s, mp));
    count_launch(2);

    NewtonParams p{};
    p.count = static_cast<int>(count);
    p.r = mp.r;
    p.c = mp.c;
    p.ld = mp.ld;
    p.O = O;
    p.ldo = ldo;
    p.strideO = strideO;
    p.otype = otype;
    p.transposed = mp.transposed;
    // blocks of 64 an accumulator: error of the result (16 x 512 x 2048, 1024 x 1024) 0.8e-6 and 0.7e-6 with one, 1.4e-6 and 1.2e-6 with two, 5.6e-6
    // and 3.8e-6 with eight, where a rounding to 16 bits is 1.7e-3 (bfloat16) or 2e-4; the FP32 iteration in one precision has 2e-6 to 5e-6
    p.core.seg = otype == OZ_F32 ? 2 : 8;
    p.core.status = mp.status;
    for (int step = 0; step < steps; ++step) {
        const double sx = plane_scale(bound[step]), ss = plane_scale(bound[step] * bound[step]),
                     sp = plane_scale(largest_polynomial(b, c, bound[step] * bound[step])), next = plane_scale(bound[step + 1]);
        const int from = step & 1;
        p.alpha = static_cast<float>(ss / (sx * sx));
        p.out = gram;
        if ((st = launch_newton<kGram>(p, map_x[from], map_x[from], s)) != OZ_OK) return st;
        p.alpha = static_cast<float>(sp * c / (ss * ss));
        p.beta = static_cast<float>(sp * b / ss);
        p.old = gram;
        p.out = poly;
        if ((st = launch_newton<kPolynomial>(p, map_s, map_s, s)) != OZ_OK) return st;
        const bool last = step == steps - 1;
        p.alpha = static_cast<float>((last ? 1.0 : next) / (sp * sx));
        p.beta = static_cast<float>((last ? 1.0 : next) * a / sx);
        p.old = x[from];
        p.out = x[from ^ 1];
        st = last ? launch_newton<kApplyLast>(p, map_p, map_x[from], s) : launch_newton<kApply>(p, map_p, map_x[from], s);
        if (st != OZ_OK) return st;
    }
    return OZ_OK;
}

}  // extern "C"
