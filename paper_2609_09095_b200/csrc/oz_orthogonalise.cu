// Orthogonalising an update by Newton-Schulz products (oz_orthogonalise): X = G / (|G|_F + eps), then a number of times
//     S = X X^T,   P = b S + c S S,   X <- a X + P X
// on the shorter side of G, which drives the singular values of X towards a common value and leaves its singular vectors.
//
// The products run on the 16-bit tensor pipe to the accuracy of FP32.  An iterate held in 16 bits would not do: what is lost in a step
// is taken up by up to |a| (3.44 with the usual coefficients) in each of the next, and the update is off by 2e-3 beyond its own
// rounding.  So a matrix is the sum of two half-precision planes hi + lo, 22 bits, of its elements times the largest power of two that
// keeps them, and 1 percent for roundings, within 2^15: hi is the rounded element, lo the rounded rest.  Of the four plane products lo lo lies below the
// last bit; the other three go into one accumulator (PLANES = 2 of the product core).  The bound of the elements lies above 2^13.9 then: those above
// 2^-17 of it keep all 22 bits, smaller ones an absolute 2^-39 of it (half of 2^-24, the step of the smallest half-precision numbers).
//
// Planes in memory: [matrix][line][chunk of 64 elements][hi, lo][64], so that both halves of an element lie at a fixed distance, and a block
// of an operand is the same box whether its lines or its elements are the inner dimension.  Elements behind the last are zero.
//
// X keeps its r rows consecutive: for X X^T it is an operand stored along its rows, for P X one stored along the inner dimension,
// both by the same bulk copies.  S and P are symmetric and computed on and below the diagonal only (see NewtonPolicy).
//
// Launches: sum of squares, planes of X, all products; narrow matrices: one.  Floor: (r r c + r r r + 2 r r c) operations a step and matrix,
// three times that on the pipe.  Five steps: 4096 x 4096 in FP32 3.6 ms, 1.15 PFLOP/s on the pipe (power cap; the FP32 iteration of a library 34);
// 16 x 512 x 2048 in bfloat16 600 us (gram on 48 of 74 pairs, 256 tiles of P X in 4 rounds); 1024 x 1024 172 us, 10 us a phase: 6.6 of them products, the rest
// storing, meeting and the first copies.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "oz_product16.cuh"

namespace oz {
namespace {

constexpr int kMaxSteps = 100;
constexpr int NORM_THREADS = 256;
constexpr int MAX_PARTS = 192;                     // partial sums of squares of a matrix
constexpr int PLANE_TILE = 64;
// Every wait of the launch of all steps, those of a block's warps for the next phase among them (a block without a tile waits with all of its
// warps while the others multiply).  The longest phase: X X^T of one row, on one pair, of as many elements as fill the memory (512 bytes of planes
// each), 350 million in 2.6 s.
constexpr unsigned long long kPhaseLimitNs = 20000000000ull;

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
    unsigned int *arrived;          // set to zero
    double eps;
    float scale;                    // of the planes
    __half *X;                      // plane pairs: [count][c][ld]
    unsigned int *status;
};

// where element i of a line of plane pairs lies; its lo half is 64 numbers on
__device__ __forceinline__ int pair_at(int i) { return (i >> 6) * 128 + (i & 63); }

// Sums of squares, in double: any finite FP32 number squares without overflow, and the order is fixed.  Columns of `column` elements are read
// 16 bytes at a time where their addresses allow.
template <class T>
__global__ void __launch_bounds__(NORM_THREADS) norm_kernel(const MatrixParams p, int64_t column, int64_t columns, int wide)
{
    __shared__ double warp_sums[NORM_THREADS / 32];
    dependency_release();
    dependency_wait();
    const int64_t matrix = blockIdx.x / p.parts;
    const int part = blockIdx.x % p.parts;
    constexpr int V = 16 / sizeof(T), UNROLL = 4;
    const T *G = static_cast<const T *>(p.G) + matrix * p.strideG;
    double sum = 0.0;
    const int64_t step = static_cast<int64_t>(p.parts) * NORM_THREADS;
    if (wide) {
        const int64_t each = (column + V - 1) / V, total = each * columns;       // pieces of V elements
        for (int64_t e0 = part * NORM_THREADS + threadIdx.x; e0 < total; e0 += UNROLL * step) {
            __align__(16) T v[UNROLL][V];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int64_t e = e0 + u * step;
                *reinterpret_cast<uint4 *>(v[u]) = make_uint4(0u, 0u, 0u, 0u);
                if (e < total) {
                    const int64_t j = total <= 0xFFFFFFFFll ? static_cast<uint32_t>(e) / static_cast<uint32_t>(each) : e / each, i = (e - j * each) * V;
                    const T *from = G + i + j * p.ldg;
                    if (i + V <= column) {
                        *reinterpret_cast<uint4 *>(v[u]) = *reinterpret_cast<const uint4 *>(from);
                    } else {
                        for (int k = 0; k < V; ++k)
                            if (i + k < column) v[u][k] = from[k];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const double x = to_float(v[u][k]);
                    sum = fma(x, x, sum);
                }
        }
    } else {
        const int64_t total = column * columns;
#pragma unroll 4
        for (int64_t e = part * NORM_THREADS + threadIdx.x; e < total; e += step) {
            const int64_t j = total <= 0xFFFFFFFFll ? static_cast<uint32_t>(e) / static_cast<uint32_t>(column) : e / column;
            const double x = to_float(G[(e - j * column) + j * p.ldg]);
            sum = fma(x, x, sum);
        }
    }
    for (int d = 16; d > 0; d /= 2) sum += __shfl_down_sync(0xFFFFFFFFu, sum, d);
    if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *p.arrived = 0u;
        for (int w = 1; w < NORM_THREADS / 32; ++w) sum += warp_sums[w];
        p.sums[blockIdx.x] = sum;
    }
}

// 1 / (|G|_F + eps) times `scale` from the sum of squares, as two factors; 0 for a matrix of zeros; NaN, which the whole update then is, for
// one that holds Inf or NaN.  The first is a power of two, so that a product with both is rounded once, and neither the number nor what it passes
// through leaves the range of FP32, from the smallest numbers to the largest.
__device__ float2 norm_factor(double sum, double eps, double scale, unsigned int *status)
{
    if (!(sum <= 1.7e308)) {
        atomicOr(status, 1u << OZ_ERR_NONFINITE_INPUT);
        return make_float2(nanf(""), 1.0f);
    }
    if (sum == 0.0) return make_float2(0.0f, 0.0f);
    const double f = scale / (sqrt(sum) + eps);
    const int half = ilogb(f) / 2;
    return make_float2(ldexpf(1.0f, half), static_cast<float>(ldexp(f, -half)));
}

// the same from a matrix' partial sums; one warp
__device__ float2 inverse_norm(const MatrixParams &p, int64_t matrix, double scale)
{
    double sum = 0.0;
    for (int i = threadIdx.x % 32; i < p.parts; i += 32) sum += p.sums[matrix * p.parts + i];
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    return norm_factor(sum, p.eps, scale, p.status);
}

// Planes of X, tiles of 64 x 64; a lane has two consecutive rows, a warp eight columns.  Through shared memory where X is the transpose of
// G.  PLANES = false: no step follows, X itself goes to O, in G's own direction.
template <class T, bool PLANES>
__global__ void __launch_bounds__(256) planes_kernel(const MatrixParams p, int tiles, int pairs)
{
    __shared__ float tile[PLANE_TILE][PLANE_TILE + 1];
    __shared__ float2 factor;
    dependency_release();
    dependency_wait();
    const uint32_t tiles_m = static_cast<uint32_t>((p.m + PLANE_TILE - 1) / PLANE_TILE);
    const uint32_t each = tiles_m * static_cast<uint32_t>((p.n + PLANE_TILE - 1) / PLANE_TILE);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    struct __align__(2 * sizeof(T)) Pair {
        T a, b;
    };
    int64_t known = -1;
    for (uint32_t item = blockIdx.x; item < static_cast<uint32_t>(tiles); item += gridDim.x) {
        const uint32_t matrix = item / each, t = item - matrix * each, tj = t / tiles_m;
        const int64_t i0 = static_cast<int64_t>(t - tj * tiles_m) * PLANE_TILE, j0 = static_cast<int64_t>(tj) * PLANE_TILE;
        const T *G = static_cast<const T *>(p.G) + matrix * p.strideG + i0 + 2 * lane + (j0 + warp) * p.ldg;
        const int rows = static_cast<int>(min(p.m - i0, static_cast<int64_t>(PLANE_TILE))) - 2 * lane;      // from the lane's first on
        const int cols = static_cast<int>(min(p.n - j0, static_cast<int64_t>(PLANE_TILE))) - warp;
        float v[8][2];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const T *from = G + 8 * s * p.ldg;
            v[s][0] = v[s][1] = 0.0f;
            if (8 * s < cols) {
                if (pairs && rows > 1) {
                    const Pair two = *reinterpret_cast<const Pair *>(from);
                    v[s][0] = to_float(two.a);
                    v[s][1] = to_float(two.b);
                } else {
                    if (rows > 0) v[s][0] = to_float(from[0]);
                    if (rows > 1) v[s][1] = to_float(from[1]);
                }
            }
        }
        __syncthreads();                                     // the tile and the factor of the round before are no longer read
        if (matrix != known) {
            if (threadIdx.x < 32) {
                const float2 f = inverse_norm(p, matrix, PLANES ? static_cast<double>(p.scale) : 1.0);
                if (threadIdx.x == 0) factor = f;
            }
            __syncthreads();
            known = matrix;
        }
        const float2 f = factor;
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int k = 0; k < 2; ++k) v[s][k] = k < rows && 8 * s < cols ? v[s][k] * f.x * f.y : 0.0f;
        if constexpr (!PLANES) {
            const int64_t at = matrix * p.strideO + i0 + 2 * lane + (j0 + warp) * p.ldo;
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (k < rows && 8 * s < cols) store_number(p.O, at + k + 8 * s * p.ldo, v[s][k], p.otype);
        } else {
            if (p.transposed) {
#pragma unroll
                for (int s = 0; s < 8; ++s)
#pragma unroll
                    for (int k = 0; k < 2; ++k) tile[warp + 8 * s][2 * lane + k] = v[s][k];
                __syncthreads();
#pragma unroll
                for (int s = 0; s < 8; ++s)
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[s][k] = tile[2 * lane + k][warp + 8 * s];
            }
            // (rows behind the last are written too: zeros)
            const int64_t x0 = p.transposed ? j0 : i0, y0 = (p.transposed ? i0 : j0) + warp;               // first row, the warp's first column of X
            __half *to = p.X + (matrix * static_cast<int64_t>(p.c) + y0) * p.ld + pair_at(static_cast<int>(x0)) + 2 * lane;
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (y0 + 8 * s < p.c) {
                    __half2 hi, lo;
                    split_planes(v[s][0], &hi.x, &lo.x);
                    split_planes(v[s][1], &hi.y, &lo.y);
                    *reinterpret_cast<__half2 *>(to + 8 * s * static_cast<int64_t>(p.ld)) = hi;
                    *reinterpret_cast<__half2 *>(to + 8 * s * static_cast<int64_t>(p.ld) + 64) = lo;
                }
        }
    }
}

template <class T>
oz_status_t launch_planes(const MatrixParams &p, bool planes, cudaStream_t stream)
{
    const bool flat = p.ldg == p.m;
    const int64_t column = flat ? p.m * p.n : p.m, columns = flat ? 1 : p.n;
    const int wide = reinterpret_cast<uintptr_t>(p.G) % 16 == 0 && (columns == 1 || p.ldg * sizeof(T) % 16 == 0) &&
                     (p.count == 1 || p.strideG * sizeof(T) % 16 == 0);
    const int pairs = reinterpret_cast<uintptr_t>(p.G) % (2 * sizeof(T)) == 0 && p.ldg % 2 == 0 && (p.count == 1 || p.strideG % 2 == 0);
    const int64_t tiles = p.count * ((p.m + PLANE_TILE - 1) / PLANE_TILE) * ((p.n + PLANE_TILE - 1) / PLANE_TILE), most = 8 * sm_count();
    if (tiles > 0x7FFFFFFF - most) return OZ_ERR_UNSUPPORTED;
    OZ_CUDA_CHECK(launch(norm_kernel<T>, dim3(static_cast<unsigned>(p.count * p.parts)), NORM_THREADS, 0, stream, p, column, columns, wide));
    OZ_CUDA_CHECK(launch(planes ? planes_kernel<T, true> : planes_kernel<T, false>, dim3(static_cast<unsigned>(tiles < most ? tiles : most)), 256, 0,
                         stream, p, static_cast<int>(tiles), pairs));
    count_launch(2);
    return OZ_OK;
}

// ---------------------------------------------------------------- products
enum { kGram, kPolynomial, kApply };

struct NewtonParams {
    int count, r, c, ld, steps;
    __half *x[2], *gram, *poly;     // plane pairs [count][c or r][ld]
    void *O;
    int64_t ldo, strideO;
    int otype, transposed;
    unsigned int *arrived;          // blocks that have finished a phase, all phases together
    Core16 core;
    float alpha[3 * kMaxSteps], beta[3 * kMaxSteps];      // of each phase: result = alpha accumulator + beta S or beta X
    float diagonal[kMaxSteps];      // of P: + diagonal I, where a X is taken in through P
};

struct NewtonMaps {
    CUtensorMap x[2], gram, poly;
};

// tiles of a matrix in a phase: all of X, or those of S and P that touch the lower blocks of 256
template <int BN>
__host__ __device__ __forceinline__ uint32_t newton_tiles(int r, int c, int phase)
{
    const uint32_t tm = static_cast<uint32_t>((r + 255) / 256), wide = 256 / BN;
    if (phase % 3 == kApply) return tm * static_cast<uint32_t>((c + BN - 1) / BN);
    const uint32_t last = (static_cast<uint32_t>(r) - 256 * (tm - 1) + BN - 1) / BN;              // columns of tiles of the last block
    return wide * tm * (tm - 1) / 2 + (tm - 1) * wide + last;
}

// (One launch a product: 283 us for 1024 x 1024 where this takes 168.)
// All steps in one launch: phase 3 s is S = X X^T of step s, 3 s + 1 P, 3 s + 2 the new X.  The blocks meet between the phases.
// Tiles are 256 rows x BN columns by pairs: the three plane products of a block read shared memory at 106 bytes a cycle with BN = 256; those of
// tiles of 128 x 128 by single CTAs would at 213 of the 128 that it has.
// Of S and P only blocks of 256 x 256 on and below the diagonal are computed and stored, line j holding elements i >= j (and all of the
// diagonal block).  A product that wants a block above takes the one below with its directions exchanged: an operand stored along its rows
// instead of along the inner dimension, which the tensor core reads as well.
// FOLDED: a X is taken in through P's diagonal, and results are 16-bit numbers (see oz_orthogonalise()).
template <bool FOLDED>
struct NewtonPolicy {
    using Params = NewtonParams;
    using Maps = NewtonMaps;
    struct Tile : Tile16 {
        int matrix, phase;
    };
    static constexpr bool RAGGED_K = false, COOPERATIVE = true;
    static constexpr unsigned long long WAIT_NS = kPhaseLimitNs;
    static constexpr int STAGING = 0;

    static __device__ __forceinline__ const CUtensorMap *map_a(const Maps &m, int phase)
    {
        return phase % 3 == kGram ? &m.x[phase / 3 & 1] : phase % 3 == kPolynomial ? &m.gram : &m.poly;
    }
    static __device__ __forceinline__ const CUtensorMap *map_b(const Maps &m, int phase)
    {
        return phase % 3 == kPolynomial ? &m.gram : &m.x[phase / 3 & 1];
    }
    static __device__ __forceinline__ void setup(const Params &, int, int *) {}
    static __device__ __forceinline__ int phases(const Params &p) { return 3 * p.steps; }

    // A block arrives with a release, cumulative over what its threads have stored before they met, and whoever goes on acquires; the proxy fences
    // carry the stores over to the bulk copies.  (Every thread with a fence of its own: 1.2 to 1.9 us.)
    static __device__ __forceinline__ bool ready(const Params &p, int phase, volatile int *abort_flag)
    {
        const unsigned int want = static_cast<unsigned int>(phase) * gridDim.x;
        unsigned long long start = 0;
        bool ok = true;
        if (threadIdx.x % 32 == 0) {
            for (unsigned int poll = 0;; ++poll) {
                unsigned int have;
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(have) : "l"(p.arrived) : "memory");
                if (have >= want) break;
                if (*abort_flag) {
                    ok = false;
                    break;
                }
                if (poll % 256 == 255) {
                    const unsigned long long now = global_timer_ns();
                    if (start == 0) start = now;
                    if (now - start > kPhaseLimitNs) {
                        *abort_flag = 1;
                        atomicOr(p.core.status, 1u << OZ_ERR_TIMEOUT);
                        ok = false;
                        break;
                    }
                }
            }
        }
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        asm volatile("fence.proxy.async;" ::: "memory");
        return ok;
    }
    static __device__ __forceinline__ void done(const Params &p, int)
    {
        asm volatile("fence.proxy.async;" ::: "memory");
        asm volatile("bar.sync 1, %0;" ::"n"(P16_EPI_WARPS * 32) : "memory");
        if (threadIdx.x == 32 * P16_FIRST_EPI) {
            __threadfence();
            asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p.arrived) : "memory");
        }
    }

    template <int CG, int BN>
    static __device__ __forceinline__ int64_t total(const Params &p, const int *, int phase)
    {
        return static_cast<int64_t>(p.count) * newton_tiles<BN>(p.r, p.c, phase);
    }

    template <int CG, int BN>
    static __device__ __forceinline__ Tile decode(const Params &p, const int *, int phase, int64_t item)
    {
        const uint32_t each = newton_tiles<BN>(p.r, p.c, phase);
        Tile t;
        t.phase = phase;
        t.matrix = static_cast<int>(static_cast<uint32_t>(item) / each);
        const uint32_t in = static_cast<uint32_t>(item) - static_cast<uint32_t>(t.matrix) * each;
        uint32_t ti, tj;
        if (phase % 3 == kApply) {
            const uint32_t tm = static_cast<uint32_t>((p.r + 255) / 256);
            ti = in % tm;
            tj = in / tm;
        } else {
            // block row ti has wide (ti + 1) tiles
            constexpr uint32_t wide = 256 / BN;
            const uint32_t block = in / wide;
            ti = static_cast<uint32_t>((sqrtf(8.0f * static_cast<float>(block) + 1.0f) - 1.0f) * 0.5f);
            while (ti * (ti + 1) / 2 > block) --ti;
            while ((ti + 1) * (ti + 2) / 2 <= block) ++ti;
            tj = in - wide * (ti * (ti + 1) / 2);
        }
        t.a_row = static_cast<int>(ti) * 256;
        t.b_row = static_cast<int>(tj) * BN;
        t.a_z = t.b_z = t.matrix;
        t.k_begin = 0;
        t.k_len = phase % 3 == kGram ? p.c : p.r;
        const int left = (phase % 3 == kApply ? p.c : p.r) - t.b_row;
        t.cols = BN > 128 && left <= 128 ? 128 : BN;
        return t;
    }

    static __device__ __forceinline__ int a_mn(const Params &, const Tile &t, int block)
    {
        return t.phase % 3 == kGram || block >> 2 <= t.a_row >> 8;
    }
    static __device__ __forceinline__ int b_mn(const Params &, const Tile &t, int block)
    {
        return t.phase % 3 == kGram || (t.phase % 3 == kPolynomial && block >> 2 < t.b_row >> 8);
    }

    // A thread has one row of X, S or P (consecutive lanes consecutive rows) and N columns, a few at a time.
    template <int CG, int BN, int N>
    static __device__ __forceinline__ void store(const Params &p, const Tile &t, const float (&acc)[N], int row, int col, unsigned char *)
    {
        const int left = (t.phase % 3 == kApply ? p.c : p.r) - t.b_row - col;
        if (left >= N) store_columns<true>(p, t, acc, t.a_row + row, t.b_row + col, left);
        else if (left > 0) store_columns<false>(p, t, acc, t.a_row + row, t.b_row + col, left);
    }

    template <bool FULL, int N>
    static __device__ __forceinline__ void store_columns(const Params &p, const Tile &t, const float (&acc)[N], int i, int j0, int left)
    {
        const bool last = t.phase == 3 * p.steps - 1;
        if (i >= (last ? p.r : p.ld / 2)) return;
        const float alpha = p.alpha[t.phase], beta = p.beta[t.phase];
        const int64_t at = (static_cast<int64_t>(t.matrix) * (t.phase % 3 == kApply ? p.c : p.r) + j0) * p.ld + pair_at(i);
        const __half *x = p.x[t.phase / 3 & 1] + at;
        if (last) {
            auto as = [&](auto *O) {
                O += t.matrix * p.strideO;
                if (p.transposed) store_last<FULL, true, !FOLDED>(p, x, O + j0 + i * p.ldo, acc, alpha, beta, left);
                else store_last<FULL, false, !FOLDED>(p, x, O + i + j0 * p.ldo, acc, alpha, beta, left);
            };
            if constexpr (!FOLDED) as(static_cast<float *>(p.O));
            else if (p.otype == OZ_BF16) as(static_cast<__nv_bfloat16 *>(p.O));
            else as(static_cast<__half *>(p.O));
        } else if (t.phase % 3 == kGram) {
            store_planes<FULL, false>(p, nullptr, p.gram + at, acc, alpha, beta, 0.0f, 0, left);
        } else if (t.phase % 3 == kPolynomial) {
            store_planes<FULL, true>(p, p.gram + at, p.poly + at, acc, alpha, beta, i < p.r ? p.diagonal[t.phase / 3] : 0.0f, i - j0, left);
        } else {
            store_planes<FULL, !FOLDED>(p, x, p.x[(t.phase / 3 & 1) ^ 1] + at, acc, alpha, beta, 0.0f, -1, left);
        }
    }

    // v = alpha acc + beta old of columns c0 .. c0 + K - 1; `old` moves on.  (Written by other blocks of this launch: from L2.)
    template <bool FULL, bool OLD, int K, int N>
    static __device__ __forceinline__ void results(float (&v)[K], const __half *&old, int64_t ld, const float (&acc)[N], int c0, float alpha,
                                                   float beta, int left)
    {
#pragma unroll
        for (int c = 0; c < K; ++c) v[c] = alpha * acc[c0 + c];
        if constexpr (OLD) {
            __half hi[K], lo[K];
#pragma unroll
            for (int c = 0; c < K; ++c) {
                const bool inside = FULL || c0 + c < left;
                hi[c] = inside ? __ldcg(old) : __half();
                lo[c] = inside ? __ldcg(old + 64) : __half();
                old += ld;
            }
#pragma unroll
            for (int c = 0; c < K; ++c) v[c] = fmaf(beta, __half2float(hi[c]) + __half2float(lo[c]), v[c]);
        }
    }

    // planes of the results, at column `on` of the thread's + diagonal
    template <bool FULL, bool OLD, int N>
    static __device__ __forceinline__ void store_planes(const Params &p, const __half *old, __half *to, const float (&acc)[N], float alpha, float beta,
                                                        float diagonal, int on, int left)
    {
        // (four with old X beside 64 running sums: eight spill 138 bytes, and 4096 x 4096 takes 3690 us instead of 3580)
        constexpr int K = OLD && !FOLDED && N >= 64 ? 4 : 8;
#pragma unroll
        for (int c0 = 0; c0 < N; c0 += K) {
            float v[K];
            results<FULL, OLD>(v, old, p.ld, acc, c0, alpha, beta, left);
#pragma unroll
            for (int c = 0; c < K; ++c) {
                if (FOLDED && OLD && c0 + c == on) v[c] += diagonal;
                if (FULL || c0 + c < left) split_planes(v[c], to, to + 64);
                to += p.ld;
            }
        }
    }

    // the results themselves: down their columns, or, transposed, the row's consecutive elements
    template <bool FULL, bool TRANSPOSED, bool OLD, int N, class T>
    static __device__ __forceinline__ void store_last(const Params &p, const __half *old, T *to, const float (&acc)[N], float alpha, float beta, int left)
    {
        const bool wide = TRANSPOSED && FULL && reinterpret_cast<uintptr_t>(to) % 16 == 0;
#pragma unroll
        for (int c0 = 0; c0 < N; c0 += 8) {
            float v[8];
            results<FULL, OLD>(v, old, p.ld, acc, c0, alpha, beta, left);
            __align__(16) T w[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) w[c] = from_float<T>(v[c]);
            if (wide) {
#pragma unroll
                for (int c = 0; c < static_cast<int>(sizeof(T)) / 2; ++c) reinterpret_cast<uint4 *>(to + c0)[c] = reinterpret_cast<const uint4 *>(w)[c];
            } else if (TRANSPOSED) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (FULL || c0 + c < left) to[c0 + c] = w[c];
            } else {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (FULL || c0 + c < left) *to = w[c];
                    to += p.ldo;
                }
            }
        }
    }
};

template <bool FOLDED, int BN>
oz_status_t launch_newton(const NewtonMaps &maps, const NewtonParams &p, cudaStream_t stream)
{
    int64_t most = 0;
    for (int phase = 0; phase < 3; ++phase) {
        const int64_t tiles = static_cast<int64_t>(p.count) * newton_tiles<BN>(p.r, p.c, phase);
        if (tiles > most) most = tiles;
    }
    if (most >= (1ll << 31)) return OZ_ERR_UNSUPPORTED;
    return launch_product16<NewtonPolicy<FOLDED>, 2, BN, 2, 1>(maps, p, most, 0, stream);
}

// cycles of a step with tiles of 256 x BN: rounds over the pairs, each with its blocks of 64 inner indices and `store` cycles for what a round
// takes besides
template <int BN>
int64_t step_cycles(const NewtonParams &p, int block, int store)
{
    int64_t sum = 0;
    for (int phase = 0; phase < 3; ++phase) {
        const int64_t tiles = static_cast<int64_t>(p.count) * newton_tiles<BN>(p.r, p.c, phase), pairs = sm_count() / 2;
        sum += (tiles + pairs - 1) / pairs * (((phase == kGram ? p.c : p.r) + 63) / 64 * block + store);
    }
    return sum;
}

// ---------------------------------------------------------------- narrow matrices
// r <= 128 and c <= 2048: a cluster of up to 8 CTAs keeps a matrix in shared memory through all steps, each CTA up to 256 of its
// columns, and one launch does everything, the norm included.  A step:
//   S   every CTA multiplies its columns, X X^T; the partial sums go to the CTA that owns a column of S, which adds them in the order
//       of the CTAs and gives its planes to all
//   P   every CTA by itself: 128 x 128 x 128
//   X   every CTA its own columns, in place: the products read all of X before the first element is written
// hi hi and the sum of the mixed products have accumulators of their own, three of hi hi in turn, added in FP32.
// Bound: latencies and two-byte accesses of shared memory, 2 to 4 us a product (launches or meetings of the whole device: 6).  128 x 512 in FP32: 71 us
// (the general form 107), 32 x 32: 20, 128 x 2048: 100 (general 177), 148 of 128 x 512: 193.
constexpr int SMALL_R = 128, SMALL_W = 256, SMALL_CTAS = 8, SMALL_THREADS = 512;
constexpr int SMALL_LINES_BYTES = SMALL_R * 128;                         // a plane of 64 elements of S or P

struct SmallParams {
    MatrixParams m;
    int steps, width;               // columns of a CTA, a multiple of 16
    int boxes_in_s;                 // no room for the partial sums beside S: two more meetings of the cluster a step
    float alpha[3 * kMaxSteps], beta[3 * kMaxSteps];
};

// byte of element i of a line, its chunk of 64 elements apart: the 128-byte swizzle of a line of 128 bytes
__device__ __forceinline__ uint32_t swizzled(int line, int i) { return static_cast<uint32_t>(line * 128 + ((((i & 63) >> 3) ^ (line & 7)) << 4) + (i & 7) * 2); }

__device__ __forceinline__ uint64_t small_desc(uint32_t addr, uint32_t leading)
{
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(leading >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}

template <class T, int CTAS>
__global__ void __launch_bounds__(SMALL_THREADS, 1) newton_small_kernel(const __grid_constant__ SmallParams p)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ double sums[SMALL_CTAS + SMALL_THREADS / 32];
    __shared__ __align__(8) unsigned long long bar_word;
    __shared__ uint32_t tmem_word;
    __shared__ int abort_word;
    const MatrixParams &m = p.m;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t place = CTAS > 1 ? cluster_ctarank() : 0u;
    const int64_t matrix = blockIdx.x / CTAS;
    const int W = p.width, r16 = (m.r + 15) / 16 * 16;
    const int first = static_cast<int>(place) * W, mine = max(0, min(W, m.c - first));            // the CTA's columns of X
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char *const X = smem_raw + (base - raw);                      // [hi, lo][chunk][W lines][128 bytes]
    const uint32_t chunk_x = static_cast<uint32_t>(W) * 128, plane_x = 2 * chunk_x;
    unsigned char *const S = X + 2 * plane_x;                              // [hi, lo][chunk][128 lines][128 bytes]
    constexpr uint32_t chunk_s = SMALL_LINES_BYTES, plane_s = 2 * chunk_s;
    const unsigned char *const boxes = p.boxes_in_s ? S : S + 2 * plane_s;
    const uint32_t x_addr = base, s_addr = base + 2 * plane_x, box_addr = s_addr + (p.boxes_in_s ? 0u : 2 * plane_s), bar = smem_u32(&bar_word);
    volatile int *abort_flag = &abort_word;

    if (tid == 0) {
        mbar_init(bar, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    dependency_wait();
    if (warp == 0) tmem_alloc<1>(smem_u32(&tmem_word), 512);

    // ---- norm: sums of squares of the CTA's columns, then of the matrix
    const T *G = static_cast<const T *>(m.G) + matrix * m.strideG;
    const int64_t step_i = m.transposed ? m.ldg : 1, step_j = m.transposed ? 1 : m.ldg;
    // the CTA's part line by line along the direction in which G is consecutive: a warp a line, eight elements of a lane (two lines' four) at a time
    const int lines = m.transposed ? m.r : mine, inner = m.transposed ? mine : m.r;
    const int64_t step_line = m.transposed ? step_i : step_j;
    const T *part_of_g = G + first * step_j;
    auto each_element = [&](auto use) {
        for (int l0 = warp; l0 < lines; l0 += 2 * (SMALL_THREADS / 32))
            for (int e0 = lane; e0 < inner; e0 += 128) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int l = l0 + u / 4 * (SMALL_THREADS / 32), e = e0 + u % 4 * 32;
                    v[u] = l < lines && e < inner ? to_float(part_of_g[l * step_line + e]) : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int l = l0 + u / 4 * (SMALL_THREADS / 32), e = e0 + u % 4 * 32;
                    if (l < lines && e < inner) use(m.transposed ? l : e, m.transposed ? e : l, v[u]);
                }
            }
    };
    double sum = 0.0;
    each_element([&](int, int, float v) { sum = fma(static_cast<double>(v), static_cast<double>(v), sum); });
    for (int d = 16; d > 0; d /= 2) sum += __shfl_down_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) sums[SMALL_CTAS + warp] = sum;
    // columns and rows that X does not have are zeros
    for (uint32_t at = tid * 16; at < 2 * plane_x; at += SMALL_THREADS * 16) *reinterpret_cast<uint4 *>(X + at) = make_uint4(0u, 0u, 0u, 0u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    dependency_release();
    const uint32_t tmem = tmem_word;
    auto meet = [&] {
        __syncwarp();
        cluster_sync_all();
    };
    if (CTAS > 1) meet();                       // the others' shared memory may be written
    if (tid == 0) {
        double all = 0.0;
        for (int w = 0; w < SMALL_THREADS / 32; ++w) all += sums[SMALL_CTAS + w];
        for (uint32_t to = 0; to < CTAS; ++to)
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(map_to_cta(smem_u32(&sums[place]), to)), "d"(all) : "memory");
    }
    if (CTAS > 1) meet();
    else __syncthreads();
    sum = 0.0;
    for (int w = 0; w < CTAS; ++w) sum += sums[w];
    const float2 f = norm_factor(sum, m.eps, static_cast<double>(m.scale), m.status);

    // ---- planes
    each_element([&](int i, int j, float v) {
        __half hi, lo;
        split_planes(v * f.x * f.y, &hi, &lo);
        unsigned char *to = X + (i >> 6) * chunk_x + swizzled(j, i);
        *reinterpret_cast<__half *>(to) = hi;
        *reinterpret_cast<__half *>(to + plane_x) = lo;
    });
    asm volatile("fence.proxy.async;" ::: "memory");
    __syncthreads();

    const int q = warp & 3, part = warp >> 2, row = q * 32 + lane;         // TMEM lanes of the warp, its quarter of the columns
    const uint32_t lanes = tmem + (static_cast<uint32_t>(q * 32) << 16);
    const bool leader = warp == 0 && elect_one();
    uint32_t phase = 0;
    // Accumulators side by side: those of hi hi, which take the pieces of the inner dimension in turn, then the mixed products'.
    // (Of 64 x 1000 in FP32 the error against 64 bits is 3.5e-6 with one of hi hi.)
    // D = A B over pieces of 16 inner indices; a plane's descriptor of piece k is its first one + k % 4 inner + k / 4 outer
    struct Operand {
        uint64_t first;
        uint32_t plane, inner, outer;
    };
    auto product = [&](uint32_t idesc, int pieces, int cols, const Operand &a, const Operand &b) {
        const uint32_t hh = cols <= 128 ? 3 : 1, wide = cols <= 128 ? 128 : 256, mixed = tmem + hh * wide;
        if (warp == 0) {
            // (the whole warp walks: descriptors stay in uniform registers)
            tc_fence_after();
            const uint32_t id = idesc | (static_cast<uint32_t>(cols >> 3) << 17);
            uint32_t turn = 0;
            for (int k = 0; k < pieces; ++k) {
                const uint64_t da = a.first + (k & 3) * a.inner + (k >> 2) * a.outer, db = b.first + (k & 3) * b.inner + (k >> 2) * b.outer;
                if (leader) {
                    umma16<1>(mixed, da + a.plane, db, id, k > 0);
                    umma16<1>(mixed, da, db + b.plane, id, 1u);
                    umma16<1>(tmem + turn * wide, da, db, id, k >= static_cast<int>(hh));
                }
                turn = turn + 1 == hh ? 0 : turn + 1;
            }
            if (leader) umma_commit<1>(bar);
        }
        __syncwarp();
        mbar_wait(bar, phase, abort_flag, m.status);
        __syncwarp();
        phase ^= 1u;
        tc_fence_after();
    };
    // after the epilogue of a product: its accumulators may be overwritten, what it stored may be multiplied
    auto finished = [&] {
        tc_fence_before();
        asm volatile("fence.proxy.async;" ::: "memory");
        __syncthreads();
    };
    // sixteen columns of a product of `cols` columns over `pieces` pieces
    auto add = [&](int col, int cols, int pieces, float (&v)[16]) {
        const int hh = cols <= 128 ? 3 : 1, wide = cols <= 128 ? 128 : 256;
        uint32_t a[16];
        tmem_ld16(lanes + hh * wide + col, a);
#pragma unroll
        for (int c = 0; c < 16; ++c) v[c] = __uint_as_float(a[c]);
        for (int h = min(hh, pieces) - 1; h >= 0; --h) {
            tmem_ld16(lanes + h * wide + col, a);
#pragma unroll
            for (int c = 0; c < 16; ++c) v[c] += __uint_as_float(a[c]);
        }
    };
    const uint32_t desc_base = idesc16(false, 1);
    const Operand x_rows{small_desc(x_addr, chunk_x), plane_x >> 4, 2048 >> 4, 4 * 2048 >> 4},     // along the rows, for X X^T
        x_lines{small_desc(x_addr, 16), plane_x >> 4, 32 >> 4, chunk_x >> 4}, s_lines{small_desc(s_addr, 16), plane_s >> 4, 32 >> 4, chunk_s >> 4};
    // the thread's row of sixteen lines of plane pairs
    auto read_pairs = [&](const unsigned char *chunk, uint32_t plane, int line, float (&v)[16]) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            const unsigned char *at = chunk + swizzled(line + c, row);
            v[c] = __half2float(*reinterpret_cast<const __half *>(at)) + __half2float(*reinterpret_cast<const __half *>(at + plane));
        }
    };
    auto write_pairs = [&](unsigned char *chunk, uint32_t plane, int line, const float (&v)[16]) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            unsigned char *at = chunk + swizzled(line + c, row);
            split_planes(v[c], reinterpret_cast<__half *>(at), reinterpret_cast<__half *>(at + plane));
        }
    };

    for (int step = 0; step < p.steps; ++step) {
        const float *alpha = p.alpha + 3 * step, *beta = p.beta + 3 * step;
        // ---- S
        const int pieces = (mine + 15) / 16;
        product(desc_base | (3u << 15), pieces, r16, x_rows, x_rows);
        if constexpr (CTAS == 1) {
#pragma unroll 1
            for (int c0 = part * 16; c0 < r16; c0 += 64) {
                float v[16];
                add(c0, r16, pieces, v);
#pragma unroll
                for (int c = 0; c < 16; ++c) v[c] *= alpha[kGram];
                if (row < r16) write_pairs(S + (row >> 6) * chunk_s, plane_s, c0, v);
            }
        } else {
            constexpr int OWN = SMALL_R / CTAS;                            // columns of S that a CTA owns; boxes [sender][column][row]
            if (p.boxes_in_s) meet();                                      // nobody multiplies with P any more
#pragma unroll 1
            for (int c0 = part * 16; c0 < r16; c0 += 64) {
                float v[16];
                if (mine > 0) {
                    add(c0, r16, pieces, v);
                } else {
#pragma unroll
                    for (int c = 0; c < 16; ++c) v[c] = 0.0f;
                }
                // (16 columns have one owner)
                const uint32_t to = map_to_cta(box_addr + static_cast<uint32_t>(((place * OWN + c0 % OWN) * SMALL_R + row) * 4), static_cast<uint32_t>(c0 / OWN));
                static_assert(OWN % 16 == 0, "owner of a piece");
                if (row < r16)
#pragma unroll
                    for (int c = 0; c < 16; ++c) store_cluster(to + c * SMALL_R * 4, v[c]);
            }
            meet();
            // two rows a thread
            constexpr int EACH = OWN / 8;
            const int own_row = 2 * (tid % 64), own_col = tid / 64;
            float2 total[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                total[e] = make_float2(0.0f, 0.0f);
                for (int s = 0; s < CTAS; ++s) {
                    const float2 v = *reinterpret_cast<const float2 *>(boxes + ((s * OWN + own_col + 8 * e) * SMALL_R + own_row) * 4);
                    total[e].x += v.x;
                    total[e].y += v.y;
                }
            }
            if (p.boxes_in_s) meet();                                      // every sum is in registers: S may be written
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int j = static_cast<int>(place) * OWN + own_col + 8 * e;
                if (j < r16 && own_row < r16) {
                    __half2 hi, lo;
                    split_planes(total[e].x * alpha[kGram], &hi.x, &lo.x);
                    split_planes(total[e].y * alpha[kGram], &hi.y, &lo.y);
                    const uint32_t to = s_addr + (own_row >> 6) * chunk_s + swizzled(j, own_row);
                    for (uint32_t cta = 0; cta < CTAS; ++cta) {
                        store_cluster(map_to_cta(to, cta), *reinterpret_cast<const float *>(&hi));
                        store_cluster(map_to_cta(to + plane_s, cta), *reinterpret_cast<const float *>(&lo));
                    }
                }
            }
            asm volatile("fence.proxy.async;" ::: "memory");
            meet();
        }
        finished();
        // ---- P
        product(desc_base, r16 / 16, r16, s_lines, s_lines);
#pragma unroll 1
        for (int c0 = part * 16; c0 < r16; c0 += 64) {
            float v[16], was[16];
            read_pairs(S + (row >> 6) * chunk_s, plane_s, c0, was);
            add(c0, r16, r16 / 16, v);
#pragma unroll
            for (int c = 0; c < 16; ++c) v[c] = fmaf(beta[kPolynomial], was[c], alpha[kPolynomial] * v[c]);
            if (row < r16) write_pairs(S + (row >> 6) * chunk_s, plane_s, c0, v);
        }
        finished();
        // ---- X
        const int cols = 16 * pieces;
        const bool last = step == p.steps - 1;
        if (mine > 0) {
            product(desc_base, r16 / 16, cols, s_lines, x_lines);
#pragma unroll 1
            for (int c0 = part * 16; c0 < cols; c0 += 64) {
                float v[16], was[16];
                unsigned char *x = X + (row >> 6) * chunk_x;
                read_pairs(x, plane_x, c0, was);
                add(c0, cols, r16 / 16, v);
#pragma unroll
                for (int c = 0; c < 16; ++c) v[c] = fmaf(beta[kApply], was[c], alpha[kApply] * v[c]);
                if (!last) {
                    if (row < r16) write_pairs(x, plane_x, c0, v);
                } else if (row < m.r) {
                    auto as = [&](auto *O) {
                        using Out = typename std::remove_pointer<decltype(O)>::type;
                        O += matrix * m.strideO + (m.transposed ? row * m.ldo + first + c0 : row + (first + c0) * m.ldo);
                        if (m.transposed && c0 + 16 <= mine && reinterpret_cast<uintptr_t>(O) % 16 == 0) {
                            // (one number at a time, a warp's 32 rows are 32 places in memory with every store)
                            __align__(16) Out w[16];
#pragma unroll
                            for (int c = 0; c < 16; ++c) w[c] = from_float<Out>(v[c]);
#pragma unroll
                            for (int c = 0; c < static_cast<int>(sizeof(Out)); ++c) reinterpret_cast<uint4 *>(O)[c] = reinterpret_cast<const uint4 *>(w)[c];
                        } else {
                            const int64_t by = m.transposed ? 1 : m.ldo;
#pragma unroll
                            for (int c = 0; c < 16; ++c)
                                if (c0 + c < mine) O[c * by] = from_float<Out>(v[c]);
                        }
                    };
                    if (m.otype == OZ_F32) as(static_cast<float *>(m.O));
                    else if (m.otype == OZ_BF16) as(static_cast<__nv_bfloat16 *>(m.O));
                    else as(static_cast<__half *>(m.O));
                }
            }
        }
        finished();
    }
    if (CTAS > 1) meet();                                                  // no CTA leaves while another may still write to it
    if (warp == 0) tmem_dealloc<1>(tmem, 512);
}

template <class T, int CTAS>
oz_status_t launch_small(const SmallParams &p, cudaStream_t stream)
{
    auto kernel = newton_small_kernel<T, CTAS>;
    const size_t smem = 1024 + 4 * static_cast<size_t>(p.width) * 128 + (CTAS == 1 || p.boxes_in_s ? 4 : 8) * SMALL_LINES_BYTES;
    static std::atomic<unsigned long long> ready{0};
    OZ_CUDA_CHECK(allow_shared(kernel, 1024 + 4 * SMALL_W * 128 + 4 * SMALL_LINES_BYTES, ready));
    static_assert(4 * 128 * 128 + 8 * SMALL_LINES_BYTES <= 4 * SMALL_W * 128 + 4 * SMALL_LINES_BYTES, "boxes of their own with up to 128 columns");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.m.count * CTAS));
    cfg.blockDim = dim3(SMALL_THREADS);
    // (more than half of a multiprocessor's: two CTAs that want all of its tensor memory never share it)
    cfg.dynamicSmemBytes = smem > 120 * 1024 ? smem : 120 * 1024;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CTAS;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    OZ_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, p));
    count_launch();
    return OZ_OK;
}

template <class T>
oz_status_t launch_small(const SmallParams &p, int ctas, cudaStream_t stream)
{
    switch (ctas) {
        case 1: return launch_small<T, 1>(p, stream);
        case 2: return launch_small<T, 2>(p, stream);
        case 4: return launch_small<T, 4>(p, stream);
        default: return launch_small<T, 8>(p, stream);
    }
}

// ---------------------------------------------------------------- host side
struct Layout {
    int64_t r, c, chunks;
    int parts;
    size_t arrived, sums, x[2], s, poly, total;
};

Layout layout_of(int64_t m, int64_t n, int64_t count)
{
    Layout l{};
    l.r = m < n ? m : n;
    l.c = m < n ? n : m;
    l.chunks = (l.r + 63) / 64;
    // pieces of 16 elements a thread, about a block a multiprocessor in all
    const int64_t pieces = (m * n + NORM_THREADS * 16 - 1) / (NORM_THREADS * 16), share = (MAX_PARTS + count - 1) / count;
    l.parts = static_cast<int>(pieces < share ? pieces : share);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += static_cast<size_t>(round_up(bytes, 256));
        return here;
    };
    l.arrived = take(4);
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

// the largest |a + b q + c q^2| of 0 <= q <= bound
double largest_polynomial(double a, double b, double c, double bound)
{
    auto value = [&](double q) { return std::fabs(a + q * (b + q * c)); };
    double most = value(0.0) > value(bound) ? value(0.0) : value(bound);
    const double q = c != 0.0 ? -b / (2.0 * c) : -1.0;
    if (q > 0.0 && q < bound && value(q) > most) most = value(q);
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
    const bool folded = otype != OZ_F32;
    for (int s = 0; s < steps; ++s) {
        bound[s + 1] = largest_value(a, b, c, bound[s]);
        const double poly = largest_polynomial(folded ? a : 0.0, b, c, bound[s] * bound[s]);
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
    mp.arrived = reinterpret_cast<unsigned int *>(ws + l.arrived);
    mp.eps = eps;
    mp.scale = static_cast<float>(plane_scale(bound[0]));
    mp.X = x[0];
    mp.status = device_status_word();
    // of each phase: result = alpha accumulator + beta S or beta X, in the scales of the planes
    float alpha[3 * kMaxSteps], beta[3 * kMaxSteps], diagonal[kMaxSteps];
    const bool small = steps > 0 && l.r <= SMALL_R && l.c <= SMALL_W * SMALL_CTAS;
    for (int step = 0; step < steps; ++step) {
        const double sx = plane_scale(bound[step]), ss = plane_scale(bound[step] * bound[step]),
                     sp = plane_scale(largest_polynomial(folded && !small ? a : 0.0, b, c, bound[step] * bound[step])),
                     next = step == steps - 1 ? 1.0 : plane_scale(bound[step + 1]);
        alpha[3 * step + kGram] = static_cast<float>(ss / (sx * sx));
        beta[3 * step + kGram] = 0.0f;
        alpha[3 * step + kPolynomial] = static_cast<float>(sp * c / (ss * ss));
        beta[3 * step + kPolynomial] = static_cast<float>(sp * b / ss);
        diagonal[step] = folded ? static_cast<float>(sp * a) : 0.0f;
        alpha[3 * step + kApply] = static_cast<float>(next / (sp * sx));
        beta[3 * step + kApply] = static_cast<float>(next * a / sx);
    }
    if (small) {
        SmallParams sp{};
        sp.m = mp;
        sp.steps = steps;
        std::copy(alpha, alpha + 3 * steps, sp.alpha);
        std::copy(beta, beta + 3 * steps, sp.beta);
        // CTAs of 128 columns while all matrices together find room on the device, of 256 at most
        int ctas = 1;
        while (ctas < SMALL_CTAS && (l.c > SMALL_W * ctas || (l.c > 128 * ctas && 2 * ctas * count <= sm_count()))) ctas *= 2;
        sp.width = static_cast<int>(round_up((l.c + ctas - 1) / ctas, 16));
        sp.boxes_in_s = sp.width > 128;
        if (count * ctas > 0x7FFFFFFF) return OZ_ERR_UNSUPPORTED;
        return type == OZ_F32 ? launch_small<float>(sp, ctas, s) : type == OZ_BF16 ? launch_small<__nv_bfloat16>(sp, ctas, s) : launch_small<__half>(sp, ctas, s);
    }
    NewtonMaps maps;
    if (steps && !(make_pair_map16(&maps.x[0], x[0], l.chunks, l.c, count) && make_pair_map16(&maps.x[1], x[1], l.chunks, l.c, count) &&
                   make_pair_map16(&maps.gram, gram, l.chunks, l.r, count) && make_pair_map16(&maps.poly, poly, l.chunks, l.r, count)))
        return OZ_ERR_CUDA;

    if (count * l.parts > 0x7FFFFFFF) return OZ_ERR_UNSUPPORTED;
    st = type == OZ_F32 ? launch_planes<float>(mp, steps > 0, s) : type == OZ_BF16 ? launch_planes<__nv_bfloat16>(mp, steps > 0, s)
                                                                                   : launch_planes<__half>(mp, steps > 0, s);
    if (st != OZ_OK) return st;
    if (steps == 0) return OZ_OK;

    NewtonParams p{};
    p.count = static_cast<int>(count);
    p.r = mp.r;
    p.c = mp.c;
    p.ld = mp.ld;
    p.steps = steps;
    p.x[0] = x[0];
    p.x[1] = x[1];
    p.gram = gram;
    p.poly = poly;
    p.O = O;
    p.ldo = ldo;
    p.strideO = strideO;
    p.otype = otype;
    p.transposed = mp.transposed;
    p.arrived = mp.arrived;
    // Blocks of 64 an accumulator.  FP32 results: error (16 x 512 x 2048, 1024 x 1024) 0.8e-6 and 0.7e-6 with one, 1.4e-6 and 1.2e-6 with two; the FP32
    // iteration in one precision has 2e-6 to 5e-6.  16-bit results: a X through P's diagonal is cut off with the sums (1024 x 1024, two blocks: 1.2e-6 -> 2.9e-6
    // before the rounding) but needs no second reading of X (245 -> 191 us when that was built).  Error before the rounding and us with one / two / four /
    // eight blocks: 1024 x 1024 1.1e-6, 203 / 2.9e-6, 183 / 6.3e-6, 173 / 1.3e-5, 168; 16 x 512 x 2048 1.1e-6, 632 / 3.0e-6, 612 / 6.8e-6, 591 / 1.5e-5, 592;
    // 2048 x 2048 1.3e-6, 558 / 3.2e-6, 494 / 7.1e-6, 494 / 1.4e-5, 494.  Four: no more than about three errors of the FP32 iteration.
    p.core.seg = otype == OZ_F32 ? 1 : 4;
    p.core.idesc = idesc16(false, 2);
    p.core.status = mp.status;
    std::copy(alpha, alpha + 3 * steps, p.alpha);
    std::copy(beta, beta + 3 * steps, p.beta);
    std::copy(diagonal, diagonal + steps, p.diagonal);
    // Cycles of a block of 64 inner indices and of a round's store and meeting, fitted to five steps of 53 sizes (at the power cap those that reach it); FP32
    // results, whose accumulators are read after every block, apart from 16-bit ones.  The pick is within 4 percent of the fastest width for all of them,
    // 0.1 in the mean (by the products' cycles alone 12 and 1.3).  us with 256 / 128 / 64 columns, the pick marked:
    //   FP32      300 x 300  197 / 138 / 121*       1024 x 1024  344 / 230 / 210*      3 x 1009 x 517  289 / 200* / 210   12 x 520 x 520  334 / 327* / 442
    //             2048 x 2048  618 / 566* / 858     16 x 512 x 2048  731* / 757 / 921  3000 x 3000  1761* / 1804 / 2659   4096 x 4096  3591* / 3902 / 6604
    //   bfloat16  300 x 300  185 / 126 / 107*       1024 x 1024  330 / 204 / 172*      3 x 1009 x 517  278 / 183 / 175*   12 x 520 x 520  295 / 267* / 340
    //             2048 x 2048  579 / 497* / 658     16 x 512 x 2048  597* / 612 / 713  3000 x 3000  1642 / 1540* / 2041   4096 x 4096  3310* / 3361 / 4910
    const int64_t wide = folded ? step_cycles<256>(p, 1600, 12000) : step_cycles<256>(p, 1520, 12400),
                  half = folded ? step_cycles<128>(p, 995, 5170) : step_cycles<128>(p, 994, 5900),
                  narrow = folded ? step_cycles<64>(p, 571, 5690) : step_cycles<64>(p, 1036, 2500);
    if (wide <= half && wide <= narrow) return folded ? launch_newton<true, 256>(maps, p, s) : launch_newton<false, 256>(maps, p, s);
    if (half <= narrow) return folded ? launch_newton<true, 128>(maps, p, s) : launch_newton<false, 128>(maps, p, s);
    return folded ? launch_newton<true, 64>(maps, p, s) : launch_newton<false, 64>(maps, p, s);
}

}  // extern "C"
