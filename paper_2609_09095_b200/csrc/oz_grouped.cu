// Products of 16-bit matrices grouped by ragged sizes (oz_gemm_grouped, oz_gemm_grouped_wgrad): the forward pass of a layer
// of experts and the gradients of its inputs and weights.
//
//   columns grouped:  C(:, j) = beta C(:, j) + op(A_g) B(:, j)                         for the columns j of group g
//   inner grouped:    C_g     = beta C_g + sum over the columns t of group g of A(:, t) B(:, t)^T
//
// The groups' offsets are on the device, written by whatever sorts the tokens, so that the tiles of a launch are counted on the
// device too: every block reads the offsets, counts the tiles of each group and walks the list of all tiles.
#include <atomic>
#include <type_traits>
#include <utility>

#include "oz_product16.cuh"

namespace oz {
namespace {

constexpr int64_t kMaxGroups = OZ_GROUPS_MAX;

struct GroupedParams {
    int64_t m, n, k;                // columns grouped: C is m x n, k the inner dimension; inner grouped: every C_g is m x n
    int64_t columns;                // what the offsets divide: n, or the columns of A and B
    int groups;
    const int64_t *offsets;
    const void *A, *B;
    // element (i, kk) of op(A_g) at g strideA + i rowA + kk innerA, element (kk, j) of B at kk innerB + j colB
    int64_t strideA, rowA, innerA, innerB, colB;
    void *C;
    int64_t ldc, strideC;
    int ctype, accumulate;
    int shared_a;                   // one A for all groups
    int a_mn;                       // A along its rows
    unsigned int *status;
    Core16 core;
};

// Where the groups begin and end, in shared memory: cuts[g] .. cuts[g + 1], and, for the form with grouped columns, how many tiles
// of `width` columns lie before each group.  All threads of the block take part.  The cuts are the offsets held to [0, columns] and to
// the largest before them: offsets out of order or range are reported, and what comes of them indexes nothing out of range.
__device__ void read_groups(const GroupedParams &p, int width, int *cuts, int *before)
{
    for (int g = threadIdx.x; g <= p.groups; g += blockDim.x) {
        const int64_t o = p.offsets[g];
        const int64_t held = o < 0 ? 0 : (o > p.columns ? p.columns : o);
        if (held != o || (g > 0 && p.offsets[g - 1] > o)) atomicOr(p.status, 1u << OZ_ERR_INVALID_ARG);
        cuts[g] = static_cast<int>(held);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int start = cuts[0], sum = 0;                    // end of the last group so far, tiles so far
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            const int g = g0 + lane;
            int end = g < p.groups ? cuts[g + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int other = __shfl_up_sync(0xFFFFFFFFu, end, d);
                if (lane >= d) end = max(end, other);
            }
            end = max(end, start);
            const int last = __shfl_up_sync(0xFFFFFFFFu, end, 1);
            const int len = end - (lane == 0 ? start : last);
            const int tiles = g < p.groups ? (len + width - 1) / width : 0;
            int upto = tiles;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int other = __shfl_up_sync(0xFFFFFFFFu, upto, d);
                if (lane >= d) upto += other;
            }
            if (g < p.groups) {
                cuts[g + 1] = end;
                if (before) before[g] = sum + upto - tiles;
            }
            sum += __shfl_sync(0xFFFFFFFFu, upto, 31);
            start = __shfl_sync(0xFFFFFFFFu, end, 31);
        }
        if (lane == 0 && before) before[p.groups] = sum;
    }
    __syncthreads();
}

// the group that tile `t` of all tiles belongs to: the last g with before[g] <= t (t < before[groups])
__device__ __forceinline__ int group_of(const int *before, int groups, int t)
{
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// c[i ldc] = acc[i] of the first `valid` columns, or the sum with what is there, rounded once either way; old values a few at a time
template <class T, bool ACCUMULATE, int N>
__device__ __forceinline__ void store_row_of(T *c, int64_t ldc, const float (&acc)[N], int valid)
{
    constexpr int STEP = N < 8 ? N : 8;
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += STEP) {
        float old[STEP];
        if constexpr (ACCUMULATE) {
            const T *from = c;
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                old[i] = i0 + i < valid ? to_float(*from) : 0.0f;
                from += ldc;
            }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            if (i0 + i < valid) *c = from_float<T>(ACCUMULATE ? old[i] + acc[i0 + i] : acc[i0 + i]);
            c += ldc;
        }
    }
}

// c[(row + i) ldc + col + j] = the j-th number of lane i, of rows below `rows` and columns below `valid`; one warp
template <class T, int N>
__device__ __forceinline__ void store_rows(T *c, int64_t ldc, const float (&acc)[N], int row, int rows, int col, int valid, unsigned char *staging)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
        __align__(16) T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = from_float<T>(acc[8 * k + e]);
        *reinterpret_cast<uint4 *>(staging + lane * 128 + ((k ^ (lane & 7)) << 4)) = *reinterpret_cast<const uint4 *>(v);
    }
    __syncwarp();
    const int chunk = lane & 7, j = col + 8 * chunk;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        const int i = 4 * s + lane / 8;
        const uint4 v = *reinterpret_cast<const uint4 *>(staging + i * 128 + ((chunk ^ (i & 7)) << 4));
        if (row + i < rows) {
            T *to = c + (row + i) * ldc + j;
            if (j + 8 <= valid) {
                *reinterpret_cast<uint4 *>(to) = v;
            } else {
                const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e < valid) reinterpret_cast<uint16_t *>(to)[e] = static_cast<uint16_t>(words[e / 2] >> (16 * (e & 1)));
            }
        }
    }
    __syncwarp();
}

// (Type and old value are told apart once a row: inside the loop that took 36 instructions an element, and 8 us a tile of 256 x 256.)
template <int N>
__device__ __forceinline__ void store_row(void *C, int64_t at, int64_t ldc, const float (&acc)[N], int valid, int ctype, int accumulate)
{
    auto as = [&](auto *c) {
        using T = typename std::remove_pointer<decltype(c)>::type;
        if (accumulate) store_row_of<T, true>(c + at, ldc, acc, valid);
        else store_row_of<T, false>(c + at, ldc, acc, valid);
    };
    if (ctype == OZ_F32) as(static_cast<float *>(C));
    else if (ctype == OZ_BF16) as(static_cast<__nv_bfloat16 *>(C));
    else as(static_cast<__half *>(C));
}

// ---------------------------------------------------------------- any alignment, without tensor cores
// A block computes tiles of 64 x 64 of C, 4 x 4 a thread, from pieces of 16 inner indices in shared memory; every operand element
// is fetched by itself, so that any leading dimension and address will do.  Bound: the FP32 pipe.
constexpr int PLAIN_TILE = 64, PLAIN_K = 16, PLAIN_THREADS = 256;

template <class T, bool INNER>
__global__ void __launch_bounds__(PLAIN_THREADS) grouped_plain_kernel(const GroupedParams p)
{
    extern __shared__ int table[];
    __shared__ float sa[PLAIN_K][PLAIN_TILE + 4], sb[PLAIN_K][PLAIN_TILE + 4];
    dependency_release();
    dependency_wait();
    int *cuts = table, *before = INNER ? nullptr : table + p.groups + 1;
    read_groups(p, PLAIN_TILE, cuts, before);
    const T *A = static_cast<const T *>(p.A), *B = static_cast<const T *>(p.B);
    const int64_t tiles_m = (p.m + PLAIN_TILE - 1) / PLAIN_TILE, tiles_n = (p.n + PLAIN_TILE - 1) / PLAIN_TILE;
    const int64_t total = INNER ? p.groups * tiles_m * tiles_n : before[p.groups] * tiles_m;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int64_t item = blockIdx.x; item < total; item += gridDim.x) {
        int g;
        int64_t i0, j0, j1, k0, k1;
        if (INNER) {
            g = static_cast<int>(item / (tiles_m * tiles_n));
            const int64_t t = item % (tiles_m * tiles_n);
            i0 = t % tiles_m * PLAIN_TILE;
            j0 = t / tiles_m * PLAIN_TILE;
            j1 = p.n;
            k0 = cuts[g];
            k1 = cuts[g + 1];
        } else {
            const int t = static_cast<int>(item / tiles_m);
            g = group_of(before, p.groups, t);
            i0 = item % tiles_m * PLAIN_TILE;
            j0 = cuts[g] + static_cast<int64_t>(t - before[g]) * PLAIN_TILE;
            j1 = cuts[g + 1];
            k0 = 0;
            k1 = p.k;
        }
        float acc[4][4] = {};
        for (int64_t kk0 = k0; kk0 < k1; kk0 += PLAIN_K) {
            // consecutive threads along the direction in which the elements lie one behind the other
#pragma unroll
            for (int e = threadIdx.x; e < PLAIN_K * PLAIN_TILE; e += PLAIN_THREADS) {
                const int ka = p.rowA == 1 ? e / PLAIN_TILE : e % PLAIN_K, ia = p.rowA == 1 ? e % PLAIN_TILE : e / PLAIN_K;
                const int kb = p.colB == 1 ? e / PLAIN_TILE : e % PLAIN_K, jb = p.colB == 1 ? e % PLAIN_TILE : e / PLAIN_K;
                sa[ka][ia] = kk0 + ka < k1 && i0 + ia < p.m
                                 ? to_float(A[g * p.strideA + (i0 + ia) * p.rowA + (kk0 + ka) * p.innerA]) : 0.0f;
                sb[kb][jb] = kk0 + kb < k1 && j0 + jb < j1 ? to_float(B[(kk0 + kb) * p.innerB + (j0 + jb) * p.colB]) : 0.0f;
            }
            __syncthreads();
#pragma unroll
            for (int kk = 0; kk < PLAIN_K; ++kk) {
                const float4 a = *reinterpret_cast<const float4 *>(&sa[kk][4 * tx]), b = *reinterpret_cast<const float4 *>(&sb[kk][4 * ty]);
                const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
            }
            __syncthreads();
        }
        if (k1 <= k0 && p.accumulate) continue;
        const int64_t col = j0 + 4 * ty;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = i0 + 4 * tx + i;
            if (row < p.m && col < j1)
                store_row(p.C, (INNER ? g * p.strideC : 0) + row + col * p.ldc, p.ldc, acc[i], static_cast<int>(min(j1 - col, static_cast<int64_t>(4))),
                          p.ctype, p.accumulate);
        }
    }
}

template <class T, bool INNER>
oz_status_t launch_plain(const GroupedParams &p, cudaStream_t stream)
{
    // enough blocks for the tiles of grouped columns that the host can count on, four of them a multiprocessor at most
    const int64_t tiles_m = (p.m + PLAIN_TILE - 1) / PLAIN_TILE, tiles_n = (p.n + PLAIN_TILE - 1) / PLAIN_TILE;
    const int64_t most = INNER ? p.groups * tiles_m * tiles_n : tiles_m * (tiles_n + p.groups);
    const int64_t grid = most < 4 * sm_count() ? most : 4 * sm_count();
    OZ_CUDA_CHECK(launch(grouped_plain_kernel<T, INNER>, dim3(static_cast<unsigned>(grid)), PLAIN_THREADS,
                         2 * (p.groups + 1) * sizeof(int), stream, p));
    count_launch();
    return OZ_OK;
}

// ---------------------------------------------------------------- tensor cores
// Bound, large products: the tensor cores at the power cap (8192 columns, 4 groups, 4096 x 4096: 192 us, 1430 TFLOP/s, where the library's product of the
// same operations takes 207 in the same run, 178 and 180 in a cooler one; tensor pipe 86 % active, operands read from memory once); few columns a
// group: memory (32 groups, 128 columns, 2048 x 4096: 90 us, 6.0 TB/s); results of short sums: the stores, five cycles a warp's store of a column (32 weight gradients 1536 x 1024 of 32 tokens: 38 us in
// FP32; in 16 bits 31, with neighbouring lanes exchanging numbers for four-byte stores 37, by rows 25).
// Rows of a tile are rows of C (features, whatever the group's size), its columns are those of a group (tokens) or of C_g: a group of
// few tokens then takes an MMA of few columns, and consecutive lanes hold consecutive elements of the column-major result.
// A group's columns are cut into equal tiles of at most BN.  The tiles that share rows of A follow one another, so that A comes from memory once.
struct GroupedMaps {
    CUtensorMap a, b;
};

// ROWS: a thread's results are consecutive elements of C instead (the operands of an inner grouped product exchanged: its rows are the columns of C), 16-bit
// numbers, 16-byte aligned.  A warp turns its 32 x 64 through shared memory and stores 128 bytes of four rows at a time.
template <bool INNER, bool ROWS = false>
struct GroupedPolicy {
    using Params = GroupedParams;
    struct Tile : Tile16 {
        int rows, valid;            // rows of C from the tile's first on, columns that belong to the group
        int64_t c;                  // element of C at the tile's first row and column
    };
    using Maps = GroupedMaps;
    static constexpr bool RAGGED_K = INNER, COOPERATIVE = false;
    static constexpr unsigned long long WAIT_NS = kWaitLimitNs;
    static constexpr int STAGING = ROWS ? P16_EPI_WARPS * 32 * 128 : 0;
    static __device__ __forceinline__ const CUtensorMap *map_a(const Maps &m, int) { return &m.a; }
    static __device__ __forceinline__ const CUtensorMap *map_b(const Maps &m, int) { return &m.b; }
    static __device__ __forceinline__ int phases(const Params &) { return 1; }
    static __device__ __forceinline__ bool ready(const Params &, int, volatile int *) { return true; }
    static __device__ __forceinline__ void done(const Params &, int) {}
    static __device__ __forceinline__ int a_mn(const Params &p, const Tile &, int) { return INNER ? 1 : p.a_mn; }
    static __device__ __forceinline__ int b_mn(const Params &, const Tile &, int) { return INNER ? 1 : 0; }

    static __device__ __forceinline__ void setup(const Params &p, int width, int *table)
    {
        read_groups(p, width, table, INNER ? nullptr : table + p.groups + 1);
    }

    template <int CG, int BN>
    static __device__ __forceinline__ int64_t total(const Params &p, const int *table, int)
    {
        const uint32_t tiles_m = static_cast<uint32_t>((p.m + 128 * CG - 1) / (128 * CG));
        if (INNER) return static_cast<int64_t>(p.groups) * tiles_m * static_cast<uint32_t>((p.n + BN - 1) / BN);
        return static_cast<int64_t>(table[2 * p.groups + 1]) * tiles_m;
    }

    // (the host sends launches of 2^31 tiles and more elsewhere: 32-bit divisions are enough)
    template <int CG, int BN>
    static __device__ __forceinline__ Tile decode(const Params &p, const int *table, int, int64_t item64)
    {
        const uint32_t item = static_cast<uint32_t>(item64), tiles_m = static_cast<uint32_t>((p.m + 128 * CG - 1) / (128 * CG));
        Tile t;
        int g, i0, j0;
        if (INNER) {
            const uint32_t tiles_n = static_cast<uint32_t>((p.n + BN - 1) / BN), each = tiles_m * tiles_n;
            g = static_cast<int>(item / each);
            const uint32_t in = item - static_cast<uint32_t>(g) * each;
            i0 = static_cast<int>(in / tiles_n) * 128 * CG;
            j0 = static_cast<int>(in % tiles_n) * BN;
            t.valid = static_cast<int>(min(static_cast<int64_t>(BN), p.n - j0));
            t.k_begin = table[g];
            t.k_len = table[g + 1] - table[g];
            t.a_z = t.b_z = 0;
            t.b_row = j0;
            t.c = g * p.strideC + (ROWS ? j0 + i0 * p.ldc : i0 + j0 * p.ldc);
        } else {
            const int *before = table + p.groups + 1;
            g = group_of(before, p.groups, static_cast<int>(item / tiles_m));
            const uint32_t in = item - static_cast<uint32_t>(before[g]) * tiles_m, tiles_n = static_cast<uint32_t>(before[g + 1] - before[g]);
            const int len = table[g + 1] - table[g], nt = static_cast<int>(in % tiles_n);
            const int width = ((len + static_cast<int>(tiles_n) - 1) / static_cast<int>(tiles_n) + 15) / 16 * 16;
            i0 = static_cast<int>(in / tiles_n) * 128 * CG;
            j0 = table[g] + nt * width;
            t.valid = min(width, table[g + 1] - j0);
            t.k_begin = 0;
            t.k_len = static_cast<int>(p.k);
            t.a_z = p.shared_a ? 0 : g;
            t.b_z = 0;
            t.b_row = j0;
            t.c = i0 + j0 * p.ldc;
        }
        t.a_row = i0;
        t.rows = static_cast<int>(p.m) - i0;
        t.cols = (t.valid + 15) / 16 * 16;
        return t;
    }

    template <int CG, int BN, int N>
    static __device__ __forceinline__ void store(const Params &p, const Tile &t, const float (&acc)[N], int row, int col, unsigned char *staging)
    {
        if constexpr (ROWS) {
            static_assert(!ROWS || N == 64, "128 bytes a row");
            if (p.ctype == OZ_BF16) store_rows(static_cast<__nv_bfloat16 *>(p.C) + t.c, p.ldc, acc, row & ~31, t.rows, col, t.valid, staging);
            else store_rows(static_cast<__half *>(p.C) + t.c, p.ldc, acc, row & ~31, t.rows, col, t.valid, staging);
            return;
        }
        if (row >= t.rows || (t.k_len == 0 && p.accumulate)) return;
        store_row(p.C, t.c + row + col * p.ldc, p.ldc, acc, t.valid - col, p.ctype, p.accumulate);
    }
};

template <bool INNER, int CG, int BN, int SPLIT = 1, bool ROWS = false>
oz_status_t launch_tiles(GroupedParams &p, bool bf16, const GroupedMaps &maps, int64_t most, cudaStream_t stream)
{
    p.core.idesc = idesc16(bf16, CG);
    return launch_product16<GroupedPolicy<INNER, ROWS>, CG, BN, 1, SPLIT>(maps, p, most, 2 * (p.groups + 1) * sizeof(int), stream);
}

// tiles of 128 cg x bn at most: what the host knows of the groups is their number and that of all columns
template <bool INNER>
int64_t most_tiles(const GroupedParams &p, int cg, int bn)
{
    const int64_t tiles_m = (p.m + 128 * cg - 1) / (128 * cg);
    if (INNER) return p.groups * tiles_m * ((p.n + bn - 1) / bn);
    const int64_t full = p.n / bn, some = p.n < p.groups ? p.n : p.groups;
    return tiles_m * (full + some);
}

// Tiles for grouped columns: those whose rounds over the multiprocessors take least.  A block of 64 inner indices costs what it moves from L2
// to shared memory, 51 to 62 bytes a cycle (pairs of 256 columns: the tensor cores, at the power cap); measured on 8 groups, 8192 columns,
// 4096 x 4096: 680, 510, 450 and 400 cycles with 256, 128, 64 and 32 columns.  A group ends in half a tile in the mean.
//   us, columns 256 / 128 / 64 / 32:  8 groups, 8192 columns, 4096 x 4096  199 / 289 / 489 / 853;  64 groups, 8192, 512 x 1024  19.6 / 22.8 / 28.8 / 40.9;
//   16 groups, 1024, 2048 x 1024  15.8 / 13.8 / 17.9 / 25.9;  16 groups, 512, 1024 x 2048  13.9 / 12.3 / 11.8 / 19.5;  8 groups, 16, 2048 x 2048
//   17.9 / 17.5 / 16.2 / 13.0.
// Tiles of 32 columns that leave most multiprocessors idle are shared by 2 or 4 along the inner dimension (one column, 4096 x 4096: 17.9 / 12.8 /
// 9.8 us with 1 / 2 / 4), where each has four blocks.
struct TileShape {
    int cg, bn, split;
};
TileShape tile_shape(const GroupedParams &p)
{
    constexpr struct {
        int cg, bn, cycles;
    } kinds[] = {{2, 256, 680}, {1, 128, 510}, {1, 64, 450}, {1, 32, 400}};
    const int64_t sms = sm_count(), some = p.n < p.groups ? p.n : p.groups, blocks = (p.k + 63) / 64;
    TileShape best{};
    int64_t least = INT64_MAX;
    for (const auto &kind : kinds) {
        const int64_t tiles_n = p.n / kind.bn + some / 2 > some ? p.n / kind.bn + some / 2 : some;
        const int64_t tiles = (p.m + 128 * kind.cg - 1) / (128 * kind.cg) * tiles_n, each = sms / kind.cg;
        const int64_t cost = (tiles + each - 1) / each * kind.cycles;
        if (cost < least) {
            least = cost;
            best = {kind.cg, kind.bn, 1};
        }
    }
    if (best.bn == 32)
        for (int split = 4; split > 1 && best.split == 1; split /= 2)
            if (most_tiles<false>(p, 1, 32) * split <= sms && blocks >= 4 * split) best.split = split;
    return best;
}

// The tensor-core form, where the operands' addresses and strides allow bulk copies; *taken says whether it did
template <bool INNER>
oz_status_t launch_tensor(GroupedParams p, oz_type_t type, bool *taken, cudaStream_t stream)
{
    *taken = false;
    bool by_rows = false;
    if constexpr (INNER) {
        // Of short sums, whose stores count more than the two stages of the ring that they take (bfloat16, numbers one by one -> by rows: 32 groups of 32,
        // 1536 x 1024, 30.7 -> 25.1 us; 16 of 256, 1024 x 2048, 24.8 -> 23.2; 16 of 512, 2048 x 2048, 62.7 -> 67.9; 16 of 1024, 4096 x 2048, 204 -> 215).
        by_rows = p.columns <= 256ll * p.groups && p.ctype != OZ_F32 && !p.accumulate && p.ldc % 8 == 0 && p.strideC % 8 == 0 && reinterpret_cast<uintptr_t>(p.C) % 16 == 0;
        if (by_rows) {
            std::swap(p.A, p.B);
            std::swap(p.m, p.n);
            std::swap(p.innerA, p.innerB);
        }
    }
    const int64_t inner = INNER ? p.columns : p.k, lda = p.rowA == 1 ? p.innerA : p.rowA, ldb = p.colB == 1 ? p.innerB : p.colB;
    if (inner == 0 || most_tiles<INNER>(p, 1, 32) >= (1ll << 31)) return OZ_OK;
    p.shared_a = INNER || p.strideA == 0 || p.groups == 1;
    if (reinterpret_cast<uintptr_t>(p.A) % 16 || reinterpret_cast<uintptr_t>(p.B) % 16 || lda % 8 || ldb % 8 || (!p.shared_a && p.strideA % 8))
        return OZ_OK;
    const bool bf16 = type == OZ_BF16;
    p.a_mn = p.rowA == 1 && p.innerA != 1;
    p.core.status = p.status;
    // Segments of 320 inner indices for FP32 results, about the error of a product that rounds every FP32 addition.  Error against 64 bits and us with
    // 256 / 320 / 384 / 512, weight gradients 2048 x 4096 of 16 experts, 16384 tokens (such a product: 2.8e-7): 2.3e-7, 273 / 2.8e-7, 268 / 3.3e-7, 265 /
    // 4.4e-7, 265; input gradients of the same (3.9e-7): 2.4e-7, 237 / 2.9e-7, 230 / 3.4e-7, 229 / 4.7e-7, 225; forward, 8192 tokens, 8 experts 4096 x
    // 4096 (6.1e-7): 2.4e-7, 229 / 2.9e-7, 217 / 3.5e-7, 214 / 4.8e-7, 214.  (The epilogue adds up every segment, and, still storing the tile before,
    // holds up the MMAs after two.)  Of 1024 for 16-bit results: 1.0e-6 before they are rounded, for a percent at most (512 / 1024 / 2048 / 4096: forward as
    // above 4.9e-7, 235 / 1.0e-6, 229 / 2.1e-6, 226 / 4.4e-6, 226; the forward pass of 128 tokens 90.0 / 89.4 / 89.0 / 88.8; sums of positive numbers,
    // which only lose, 2.2e-6 with 1024 and 1.4e-5 with 4096, in half precision, whose products are cut off one by one, 6.1e-6 and 2.6e-5).
    p.core.seg = p.ctype == OZ_F32 ? 5 : 16;
    const TileShape shape = INNER ? TileShape{2, 256, 1} : tile_shape(p);
    GroupedMaps maps;
    const int64_t za = p.shared_a ? 1 : p.groups;
    const int boxB = shape.bn < 64 ? shape.bn : 64;
    if (!(p.a_mn ? make_map16(&maps.a, bf16, p.A, p.m, inner, lda, za, za > 1 ? p.strideA : lda, 64)
                      : make_map16(&maps.a, bf16, p.A, inner, p.m, lda, za, za > 1 ? p.strideA : lda, 64)) ||
        !(INNER ? make_map16(&maps.b, bf16, p.B, p.n, inner, ldb, 1, ldb, boxB) : make_map16(&maps.b, bf16, p.B, inner, p.n, ldb, 1, ldb, boxB)))
        return OZ_OK;
    *taken = true;
    const int64_t most = most_tiles<INNER>(p, shape.cg, shape.bn);
    if constexpr (!INNER) {
        if (shape.bn == 128) return launch_tiles<INNER, 1, 128>(p, bf16, maps, most, stream);
        if (shape.bn == 64) return launch_tiles<INNER, 1, 64>(p, bf16, maps, most, stream);
        if (shape.bn == 32)
            return shape.split == 4   ? launch_tiles<INNER, 1, 32, 4>(p, bf16, maps, most, stream)
                   : shape.split == 2 ? launch_tiles<INNER, 1, 32, 2>(p, bf16, maps, most, stream)
                                      : launch_tiles<INNER, 1, 32>(p, bf16, maps, most, stream);
    }
    if constexpr (INNER)
        if (by_rows) return launch_tiles<true, 2, 256, 1, true>(p, bf16, maps, most, stream);
    return launch_tiles<INNER, 2, 256>(p, bf16, maps, most, stream);
}

// ---------------------------------------------------------------- checks that both entry points share
bool aligned_to(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

size_t size_of_type(int type) { return type == OZ_F32 ? 4 : 2; }

oz_status_t check_types(oz_type_t type, oz_type_t ctype, double beta, const void *A, const void *B, const void *C)
{
    if ((type != OZ_BF16 && type != OZ_F16) || (ctype != type && ctype != OZ_F32)) return OZ_ERR_INVALID_ARG;
    if (!aligned_to(A, 2) || !aligned_to(B, 2) || !aligned_to(C, size_of_type(ctype))) return OZ_ERR_INVALID_ARG;
    return beta == 0.0 || beta == 1.0 ? OZ_OK : OZ_ERR_UNSUPPORTED;
}

template <bool INNER>
oz_status_t launch_grouped(GroupedParams &p, oz_type_t type, cudaStream_t stream)
{
    oz_status_t st = ensure_device_ready();
    if (st != OZ_OK) return st;
    p.status = device_status_word();
    bool taken = false;
    st = launch_tensor<INNER>(p, type, &taken, stream);
    if (taken || st != OZ_OK) return st;
    return type == OZ_BF16 ? launch_plain<__nv_bfloat16, INNER>(p, stream) : launch_plain<__half, INNER>(p, stream);
}

}  // namespace
}  // namespace oz

using namespace oz;

extern "C" {

oz_status_t oz_gemm_grouped(int transA, int64_t m, int64_t n, int64_t k, int64_t groups, const int64_t *offsets,
                            oz_type_t type, const void *A, int64_t lda, int64_t strideA, const void *B, int64_t ldb,
                            oz_type_t ctype, double beta, void *C, int64_t ldc, void *stream)
{
    if (m < 0 || n < 0 || k < 0 || groups < 0 || strideA < 0 || (transA != 0 && transA != 1)) return OZ_ERR_INVALID_ARG;
    oz_status_t st = check_types(type, ctype, beta, A, B, C);
    if (st != OZ_OK) return st;
    if (m > OZ_EXTENT_MAX || n > OZ_EXTENT_MAX || k > OZ_EXTENT_MAX || groups > kMaxGroups) return OZ_ERR_UNSUPPORTED;
    if (m == 0 || n == 0 || groups == 0) return OZ_OK;
    if (!offsets || !aligned_to(offsets, 8) || !C || ldc < m) return OZ_ERR_INVALID_ARG;
    if (k > 0 && (!A || !B || lda < (transA ? k : m) || ldb < k)) return OZ_ERR_INVALID_ARG;
    if (k == 0 && beta == 1.0) return OZ_OK;
    GroupedParams p{};
    p.m = m;
    p.n = p.columns = n;
    p.k = k;
    p.groups = static_cast<int>(groups);
    p.offsets = offsets;
    p.A = A;
    p.B = B;
    p.strideA = strideA;
    p.rowA = transA ? lda : 1;
    p.innerA = transA ? 1 : lda;
    p.innerB = 1;
    p.colB = ldb;
    p.C = C;
    p.ldc = ldc;
    p.ctype = ctype;
    p.accumulate = beta == 1.0;
    return launch_grouped<false>(p, type, static_cast<cudaStream_t>(stream));
}

oz_status_t oz_gemm_grouped_wgrad(int64_t m, int64_t n, int64_t tokens, int64_t groups, const int64_t *offsets,
                                  oz_type_t type, const void *A, int64_t lda, const void *B, int64_t ldb, oz_type_t ctype,
                                  double beta, void *C, int64_t ldc, int64_t strideC, void *stream)
{
    if (m < 0 || n < 0 || tokens < 0 || groups < 0) return OZ_ERR_INVALID_ARG;
    oz_status_t st = check_types(type, ctype, beta, A, B, C);
    if (st != OZ_OK) return st;
    if (m > OZ_EXTENT_MAX || n > OZ_EXTENT_MAX || tokens > OZ_EXTENT_MAX || groups > kMaxGroups) return OZ_ERR_UNSUPPORTED;
    if (m == 0 || n == 0 || groups == 0) return OZ_OK;
    if (!offsets || !aligned_to(offsets, 8) || !C || ldc < m) return OZ_ERR_INVALID_ARG;
    if (groups > 1 && (strideC < m || (strideC - m) / ldc < n - 1)) return OZ_ERR_INVALID_ARG;
    if (tokens > 0 && (!A || !B || lda < m || ldb < n)) return OZ_ERR_INVALID_ARG;
    GroupedParams p{};
    p.m = m;
    p.n = n;
    p.columns = tokens;
    p.groups = static_cast<int>(groups);
    p.offsets = offsets;
    p.A = A;
    p.B = B;
    p.rowA = 1;
    p.innerA = lda;
    p.innerB = ldb;
    p.colB = 1;
    p.C = C;
    p.ldc = ldc;
    p.strideC = strideC;
    p.ctype = ctype;
    p.accumulate = beta == 1.0;
    return launch_grouped<true>(p, type, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
