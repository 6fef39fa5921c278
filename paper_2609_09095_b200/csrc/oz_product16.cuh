// The core of the products of 16-bit matrices: tiles of D = A B on the 5th-generation tensor cores (kind::f16, FP32 accumulation in
// tensor memory), for operands stored along either direction.  What a tile is, how many there are and where its result goes is a
// policy's (grouped products, Newton-Schulz products).
//
// A tile is 128 CG rows x BN columns (CG = 2: a pair of CTAs shares one tcgen05.mma.cta_group::2, each CTA holds its own 128 rows
// of A, half of the columns of B and the accumulators of its rows).  The inner dimension comes in blocks of 64 elements, 128 bytes:
//   K-major operand:  boxes of 64 rows, 128 bytes of K each
//   MN-major operand: boxes of 64 inner indices, 128 bytes of consecutive rows each
// both 8 KiB, 128-byte swizzle; out-of-range elements are read as zero.
//
// PLANES = 2: an operand is the sum of two 16-bit planes hi + lo; a stage holds both of A and both of B, and a block takes the three
// products lo hi, hi lo, hi hi into one accumulator (lo lo is below the last bit of what the planes keep).
//
// Accumulation.  The tensor core cuts its running sum off at 24 bits with every instruction, 16 inner indices, which on long sums costs
// bits that FP32 results would show.  So the sum is cut into segments of seg blocks, each with an accumulator of its own
// (two slots in turn), which the epilogue warps add up in registers, rounding to nearest.
//
// A persistent CTA of 19 warps per multiprocessor:
//   warp 0       bulk copies into a ring of shared memory (no multicast)
//   warp 1       issues the MMAs (of a pair: the leader's)
//   warp 2       RAGGED_K (pairs only): zeroes, in the last block of a tile, the inner indices that belong to the next group, in both
//                operands (zeroing one would leave 0 x NaN)
//   warps 3..18  epilogue, four per lane quarter of the tensor memory, BN / 4 columns each
//
// SPLIT > 1: products of so few tiles that most multiprocessors would have none.  A cluster of SPLIT single CTAs shares one tile, each
// member a range of the inner dimension; at the end every member owns BN / SPLIT columns, gets the others' sums of them through shared
// memory of the cluster (in the ring, which nothing fills any more), adds them in the order of the members and stores.  One tile a cluster.
//
// Every wait is bounded: when one runs out the CTA reports OZ_ERR_TIMEOUT, leaves its loops, frees its tensor memory and returns.
//
// The tensor memory is taken after dependency_wait() and the successor let in after that: a CTA that waits for its predecessor
// holds none of what the predecessor still has to take.  (Cooperative launches neither wait nor let in.)
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "oz_tcgen05.cuh"

namespace oz {

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_float(float v) { return v; }

constexpr int P16_THREADS = 19 * 32;
constexpr int P16_FIRST_EPI = 3;
constexpr int P16_EPI_WARPS = 16;
constexpr int P16_BLOCK_K = 64;                    // elements: 128 bytes
constexpr int P16_BOX_BYTES = 64 * 128;
constexpr int P16_RING_BYTES = 192 * 1024;
constexpr int P16_BARRIER_BYTES = 512;

template <int CG, int BN, int PLANES, int STAGING>
struct Ring16 {
    static_assert(P16_EPI_WARPS * 4 * 32 * (BN / 4) <= P16_RING_BYTES, "sums of the other members of a cluster");
    static constexpr int B_ROWS = BN / CG;                                   // columns of the tile that one CTA loads
    static constexpr int B_BOX_ROWS = B_ROWS < 64 && PLANES == 1 ? B_ROWS : 64;
    static constexpr int B_BOXES = B_ROWS < 64 ? 1 : B_ROWS / 64;
    static constexpr int B_BOX_BYTES = B_BOX_ROWS * 128;
    static constexpr int A_PLANE = 2 * P16_BOX_BYTES;
    static constexpr int B_PLANE = B_BOXES * B_BOX_BYTES;
    static constexpr int STAGE = PLANES * (A_PLANE + B_PLANE);
    static constexpr int STAGES = (P16_RING_BYTES - STAGING) / STAGE;
    static constexpr int COLS = BN / 4;                                      // columns of an epilogue warp
    static_assert(24 * STAGES + 48 <= P16_BARRIER_BYTES, "barriers");
};

// what the roles need to know of a launch and of a tile, whatever the policy
struct Core16 {
    uint32_t idesc;             // instruction descriptor without directions and number of columns
    int seg;                    // blocks per accumulator
    unsigned int *status;
};
struct Tile16 {
    int a_row, a_z, b_row, b_z; // coordinates of the tile's first row of A and column of B
    int k_begin, k_len;
    int cols;                   // columns computed: a multiple of 16, for pairs too; of plane pairs, whose operand B may be along its rows, 64 or a multiple of 128
};

__host__ __device__ inline uint32_t idesc16(bool bf16, int cg)
{
    const uint32_t fmt = bf16 ? 1u : 0u;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | (static_cast<uint32_t>((128 * cg) >> 4) << 24);
}

template <int CG>
__device__ __forceinline__ void umma16(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}

// shared-memory descriptor of a plane of an operand.  K-major: groups of 8 rows 1024 bytes apart.  MN-major: groups of 8 inner
// indices 1024 bytes apart (stride), the next 64 rows in the next box (leading).
__device__ __forceinline__ uint64_t smem_desc16(uint32_t addr, int mn)
{
    const uint64_t leading = mn ? P16_BOX_BYTES >> 4 : 1;
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (leading << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// A wait for something that may be many tiles away: it ends with the others' waits, which are for the next block or tile, or after thirty times their limit.
__device__ __forceinline__ bool mbar_wait_rare(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned int *status)
{
    const unsigned long long start = global_timer_ns();
    for (;;) {
#pragma unroll 1
        for (int it = 0; it < 256; ++it)
            if (mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        if (global_timer_ns() - start > 30 * kWaitLimitNs) {
            *abort_flag = 1;
            atomicOr(status, 1u << OZ_ERR_TIMEOUT);
            return false;
        }
    }
}

// arrivals at a barrier of any CTA of the cluster, ordered after this thread's (and, through it, its warp's) writes
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// (relaxed: the thread has written nothing that the waiter reads, and a release would wait for a fence of the whole cluster with
// every stage: 1570 cycles a block of 256 x 256 x 64 instead of the tensor cores' 512)
__device__ __forceinline__ void mbar_expect_tx_cluster(uint32_t cluster_addr, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(cluster_addr), "r"(bytes) : "memory");
}

__device__ __forceinline__ void store_cluster(uint32_t cluster_addr, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}

// 64 elements x 64 lines of a plane of a matrix in plane pairs: (element, chunk and plane, line, matrix)
__device__ __forceinline__ void tma_load_4d_pair(uint32_t dst, const CUtensorMap *map, uint32_t bar_cluster, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// Policy P:
//   P::Params              the launch: has a Core16 `core`
//   P::Maps                the operands' maps; P::map_a(maps, phase), P::map_b(maps, phase) point to them
//   P::Tile                a tile: derives from Tile16
//   P::RAGGED_K            k_begin and k_len are any numbers, and what lies behind them must not enter (MN-major operands only)
//   P::setup(p, width, table)   all threads, after the predecessor's end: what `table`, shared memory of the launch's choice, holds
//   P::phases(p)           products that follow one another in the launch, each of results of the one before
//   P::ready(p, phase, abort_flag)   the copying warp, before its first access to what the phase before wrote; false: give up
//   P::done(p, phase)      the epilogue warps, after their last store of a phase
//   P::total<CG, BN>(p, table, phase)   number of tiles
//   P::decode<CG, BN>(p, table, phase, item)
//   P::a_mn(p, tile, block), P::b_mn(p, tile, block): whether the operand of the tile's block is stored along its rows (MN-major)
//   P::STAGING             bytes of shared memory, off the ring, through which store() takes its results: a sixteenth an epilogue warp
//   P::COOPERATIVE         the launch's blocks wait for one another (between phases)
//   P::WAIT_NS             limit of a wait: longer than a tile's next step takes and, between phases, than the other blocks' tiles
//   P::store<CG, BN>(p, tile, acc, row, col, staging): the thread's results, row of the tile (0 .. 128 CG - 1), as many columns from col on as acc
//                          holds; called by whole warps
template <class P, int CG, int BN, int PLANES, int SPLIT>
__global__ void __launch_bounds__(P16_THREADS, 1)
product16_kernel(const __grid_constant__ typename P::Maps maps, const __grid_constant__ typename P::Params p)
{
    using R = Ring16<CG, BN, PLANES, P::STAGING>;
    constexpr int STAGES = R::STAGES;
    constexpr int TMEM_COLUMNS = 2 * BN;
    static_assert(CG == 2 ? SPLIT == 1 : (PLANES == 1 && !P::RAGGED_K), "single CTAs share tiles; pairs have plane pairs and ragged ends");
    const uint32_t place = CG * SPLIT > 1 ? cluster_ctarank() : 0u;
    const uint32_t rank = CG == 2 ? place : 0u;                     // in the pair, whose first CTA leads
    const int member = CG == 2 ? 0 : static_cast<int>(place);       // of the SPLIT that share a tile
    const int64_t first_item = blockIdx.x / (CG * SPLIT);
    const int64_t item_step = gridDim.x / (CG * SPLIT);
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    const uint32_t full_bar = ring + P16_RING_BYTES;            // STAGES x 8 bytes each
    const uint32_t empty_bar = full_bar + 8 * STAGES;
    const uint32_t tail_bar = empty_bar + 8 * STAGES;
    const uint32_t tfull_bar = tail_bar + 8 * STAGES;           // 2 x 8
    const uint32_t tempty_bar = tfull_bar + 16;                 // 2 x 8
    const uint32_t go_bar = tempty_bar + 16;                    // 8: a phase may be read
    unsigned char *gen = smem_raw + (ring - raw) + P16_RING_BYTES;
    volatile uint32_t *tmem_base_ptr = reinterpret_cast<volatile uint32_t *>(gen + 24 * STAGES + 40);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gen + 24 * STAGES + 44);
    int *table = reinterpret_cast<int *>(gen + P16_BARRIER_BYTES);
    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        prefetch_map(P::map_a(maps, 0));
        prefetch_map(P::map_b(maps, 0));
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar + 8 * s, CG);                    // a CTA's copies, or what zeroes behind them, arrive once
            mbar_init(empty_bar + 8 * s, 1);
            mbar_init(tail_bar + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(tfull_bar + 8 * s, 1);
            mbar_init(tempty_bar + 8 * s, P16_EPI_WARPS * CG);
        }
        mbar_init(go_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (!P::COOPERATIVE) dependency_wait();
    if (warp == 1) tmem_alloc<CG>(smem_u32(const_cast<uint32_t *>(tmem_base_ptr)), TMEM_COLUMNS);
    P::setup(p, BN, table);
    tc_fence_before();
    __syncthreads();
    if (CG * SPLIT > 1) cluster_sync_all();   // the peers' barriers exist before anything signals them
    tc_fence_after();
    if (!P::COOPERATIVE) dependency_release();
    const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, *tmem_base_ptr, 0);
    unsigned int *const status = p.core.status;
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, abort_flag, status, P::WAIT_NS)) != 0; };
    // the member's blocks of a tile
    auto first_block = [&](int blocks) { return SPLIT == 1 ? 0 : static_cast<int>(static_cast<int64_t>(blocks) * member / SPLIT); };
    auto end_block = [&](int blocks) { return SPLIT == 1 ? blocks : static_cast<int>(static_cast<int64_t>(blocks) * (member + 1) / SPLIT); };
    auto needs_tail = [&](const Tile16 &t) { return P::RAGGED_K && (t.k_len & 15) != 0; };

    if (warp < P16_FIRST_EPI) {
        // whole warps walk the loops, one elected lane issues: addresses and descriptors stay in uniform registers
        const bool leader = elect_one();
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        if (warp == 0) {
            // -------------------------------------------------------- copies
            for (int ph = 0, phases = P::phases(p); ok && ph < phases; ++ph) {
            if (ph > 0) {
                // one warp of a block asks for the others' arrival: all of them asking keep the arrivals from getting through
                ok = P::ready(p, ph, abort_flag);
                if (!ok) break;
                if (leader) mbar_arrive(go_bar);
            }
            const CUtensorMap *mapA = P::map_a(maps, ph), *mapB = P::map_b(maps, ph);
            const int64_t total = P::template total<CG, BN>(p, table, ph);
            for (int64_t item = first_item; ok && item < total; item += item_step) {
                const typename P::Tile t = P::template decode<CG, BN>(p, table, ph, item);
                const int blocks = (t.k_len + P16_BLOCK_K - 1) / P16_BLOCK_K;
                const int b_rows = t.cols / CG, b_boxes = R::B_BOXES == 1 ? 1 : (b_rows + 63) >> 6;
                const int a_row = t.a_row + static_cast<int>(rank) * 128, b_row = t.b_row + static_cast<int>(rank) * b_rows;
                const uint32_t bytes = PLANES * (R::A_PLANE + b_boxes * R::B_BOX_BYTES);
                for (int kb = first_block(blocks), end = end_block(blocks); ok && kb < end; ++kb) {
                    ok = wait(empty_bar + 8 * stage, phase ^ 1u);
                    if (!ok) break;
                    const int kk = t.k_begin + kb * P16_BLOCK_K;
                    const uint32_t sa = ring + stage * R::STAGE, sb = sa + PLANES * R::A_PLANE;
                    const bool tail = needs_tail(t) && kb == blocks - 1;
                    if (leader) {
                        uint32_t bar;
                        if (CG == 1) {
                            bar = full_bar + 8 * stage;
                            mbar_expect_tx(bar, bytes);
                        } else {
                            bar = tail ? map_to_cta(tail_bar + 8 * stage, rank) : map_to_cta(full_bar + 8 * stage, 0u);
                            mbar_expect_tx_cluster(bar, bytes);
                        }
                        const int a_mn = P::a_mn(p, t, kb), b_mn = P::b_mn(p, t, kb);
                        auto copy = [&](uint32_t dst, const CUtensorMap *map, int mn, int row, int z, int plane) {
                            const int c0 = mn ? row : kk, c1 = mn ? kk : row;
                            if constexpr (PLANES == 2) {
                                tma_load_4d_pair(dst, map, bar, c0 & 63, 2 * (c0 >> 6) + plane, c1, z);
                            } else {
                                if (CG == 1) tma_load_3d(dst, map, bar, c0, c1, z);
                                else tma_load_3d_pair(dst, map, bar, c0, c1, z);
                            }
                        };
#pragma unroll
                        for (int pl = 0; pl < PLANES; ++pl) {
#pragma unroll
                            for (int b = 0; b < 2; ++b)
                                copy(sa + pl * R::A_PLANE + b * P16_BOX_BYTES, mapA, a_mn, a_row + 64 * b, t.a_z, pl);
#pragma unroll
                            for (int b = 0; b < R::B_BOXES; ++b)
                                if (b < b_boxes) copy(sb + pl * R::B_PLANE + b * R::B_BOX_BYTES, mapB, b_mn, b_row + 64 * b, t.b_z, pl);
                        }
                    }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            }
        } else if (warp == 1 && rank == 0) {
            // -------------------------------------------------------- MMAs
            int slot = 0;
            uint32_t slot_phase = 0;
            for (int ph = 0, phases = P::phases(p); ok && ph < phases; ++ph) {
            const int64_t total = P::template total<CG, BN>(p, table, ph);
            for (int64_t item = first_item; ok && item < total; item += item_step) {
                const typename P::Tile t = P::template decode<CG, BN>(p, table, ph, item);
                const int blocks = (t.k_len + P16_BLOCK_K - 1) / P16_BLOCK_K;
                for (int kb0 = first_block(blocks), end = end_block(blocks); ok && kb0 < end; kb0 += p.core.seg) {
                    ok = wait(tempty_bar + 8 * slot, ((slot_phase >> slot) & 1u) ^ 1u);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + static_cast<uint32_t>(slot * BN);
                    const int kb1 = min(end, kb0 + p.core.seg);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        ok = wait(full_bar + 8 * stage, phase);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t sa = ring + stage * R::STAGE, sb = sa + PLANES * R::A_PLANE;
                        const int a_mn = P::a_mn(p, t, kb), b_mn = P::b_mn(p, t, kb);
                        const uint64_t a = smem_desc16(sa, a_mn), b = smem_desc16(sb, b_mn);
                        const uint32_t step_a = a_mn ? 2048 >> 4 : 32 >> 4, step_b = b_mn ? 2048 >> 4 : 32 >> 4;      // 16 inner indices on
                        const uint32_t idesc = p.core.idesc | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) |
                                               (static_cast<uint32_t>(t.cols >> 3) << 17);
                        const int left = t.k_len - kb * P16_BLOCK_K;
                        if (leader) {
                            if constexpr (PLANES == 2) {
                                constexpr uint64_t a_lo = R::A_PLANE >> 4, b_lo = R::B_PLANE >> 4;
#pragma unroll
                                for (int ks = 0; ks < 4; ++ks)
                                    if (ks * 16 < left) {
                                        umma16<CG>(d, a + a_lo + ks * step_a, b + ks * step_b, idesc, kb > kb0 || ks > 0 ? 1u : 0u);
                                        umma16<CG>(d, a + ks * step_a, b + b_lo + ks * step_b, idesc, 1u);
                                    }
#pragma unroll
                                for (int ks = 0; ks < 4; ++ks)
                                    if (ks * 16 < left) umma16<CG>(d, a + ks * step_a, b + ks * step_b, idesc, 1u);
                            } else {
#pragma unroll
                                for (int ks = 0; ks < 4; ++ks)
                                    if (ks * 16 < left) umma16<CG>(d, a + ks * step_a, b + ks * step_b, idesc, kb > kb0 || ks > 0 ? 1u : 0u);
                            }
                            umma_commit<CG>(empty_bar + 8 * stage);
                        }
                        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    if (leader) umma_commit<CG>(tfull_bar + 8 * slot);
                    slot_phase ^= 1u << slot;
                    slot ^= 1;
                }
            }
            }
        } else if (P::RAGGED_K && warp == 2) {
            // -------------------------------------------------------- inner indices behind the group's end
            // One warp, all tiles in order: each wait is for the next phase of its barrier.  (Of two warps in turns one would wait for the phase after it
            // where two tiles end in the same stage, and a wait on a parity returns at once while the phase before is open.)
            uint32_t tail_phase = 0;                         // bit s: phase of stage s's tail barrier
            const int64_t total = P::template total<CG, BN>(p, table, 0);
            for (int64_t item = first_item; ok && item < total; item += item_step) {
                const typename P::Tile t = P::template decode<CG, BN>(p, table, 0, item);
                const int blocks = (t.k_len + P16_BLOCK_K - 1) / P16_BLOCK_K;
                const int last = (stage + blocks - 1) % STAGES;
                stage = (stage + blocks) % STAGES;
                if (!needs_tail(t)) continue;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait_rare(tail_bar + 8 * last, (tail_phase >> last) & 1u, abort_flag, status)) != 0;
                if (!ok) break;
                tail_phase ^= 1u << last;
                const int from = t.k_len & 63, to = (from + 15) & ~15;
                const int boxes = 2 + (t.cols / CG + 63) / 64;
                static_assert(!P::RAGGED_K || (PLANES == 1 && R::B_BOX_ROWS == 64), "ragged inner dimension: one plane, whole boxes");
                // a row of a box is one inner index: its eight chunks of 16 bytes stay in the row under the swizzle
                unsigned char *first = smem_raw + (ring - raw) + last * R::STAGE + (from + lane / 8) * 128 + lane % 8 * 16;
                for (int box = 0; box < boxes; ++box)
#pragma unroll
                    for (int row = 0; row < 16; row += 4)
                        if (from + lane / 8 + row < to) *reinterpret_cast<uint4 *>(first + box * P16_BOX_BYTES + row * 128) = make_uint4(0u, 0u, 0u, 0u);
                asm volatile("fence.proxy.async;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(full_bar + 8 * last, 0u));
            }
        }
        if (!ok) {
            // give copies and MMAs in flight a bounded time to land before the CTA exits
            const unsigned long long t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 2000000ull) { }
        }
    }
    // ---------------------------------------------------------------- epilogue
    constexpr int W = R::COLS < 16 ? 8 : 16;                 // columns of a load: the running sums and these stay within the registers
    const int q = warp & 3;                                  // lane quarter of the tensor memory
    const int part = (warp - P16_FIRST_EPI) >> 2;            // BN / 4 of the tile's columns
    unsigned char *const staging = smem_raw + (ring - raw) + (P16_RING_BYTES - P::STAGING) + (warp - P16_FIRST_EPI) * (P::STAGING / P16_EPI_WARPS);
    float acc[R::COLS];
    // the tile's sums (of the member's blocks)
    int slot = 0;
    uint32_t slot_phase = 0;
    auto collect = [&](const Tile16 &t) {
        const int blocks = (t.k_len + P16_BLOCK_K - 1) / P16_BLOCK_K;
#pragma unroll
        for (int c = 0; c < R::COLS; ++c) acc[c] = 0.0f;
        for (int kb0 = first_block(blocks), end = end_block(blocks); kb0 < end; kb0 += p.core.seg) {
            if (!wait(tfull_bar + 8 * slot, (slot_phase >> slot) & 1u)) return false;
            tc_fence_after();
            const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(slot * BN + part * R::COLS);
#pragma unroll
            for (int c0 = 0; c0 < R::COLS; c0 += W) {
                if (part * R::COLS + c0 >= t.cols) break;
                uint32_t v[W];
                if constexpr (W == 16) tmem_ld16(taddr + c0, v);
                else tmem_ld8(taddr + c0, v);
#pragma unroll
                for (int c = 0; c < W; ++c) acc[c0 + c] += __uint_as_float(v[c]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) mbar_arrive_relaxed(tempty_bar + 8 * slot);
                else mbar_arrive_cluster_relaxed(map_to_cta(tempty_bar + 8 * slot, 0u));
            }
            slot_phase ^= 1u << slot;
            slot ^= 1;
        }
        return true;
    };
    if constexpr (SPLIT == 1) {
        if (warp >= P16_FIRST_EPI) {
            // (a warp that has given up goes through the phases all the same: done() is where the warps of a block meet)
            bool ok = true;
            for (int ph = 0, phases = P::phases(p); ph < phases; ++ph) {
                if (ph > 0) ok = ok && wait(go_bar, (ph & 1) ^ 1);
                const int64_t total = P::template total<CG, BN>(p, table, ph);
                for (int64_t item = first_item; ok && item < total; item += item_step) {
                    const typename P::Tile t = P::template decode<CG, BN>(p, table, ph, item);
                    ok = collect(t);
                    if (ok) P::template store<CG, BN>(p, t, acc, static_cast<int>(rank) * 128 + q * 32 + lane, part * R::COLS, staging);
                }
                P::done(p, ph);
            }
        }
    } else {
        constexpr int OWN = R::COLS / SPLIT;
        const bool works = warp >= P16_FIRST_EPI && first_item < P::template total<CG, BN>(p, table, 0);
        typename P::Tile t;
        bool ok = works;
        if (works) {
            t = P::template decode<CG, BN>(p, table, 0, first_item);
            ok = collect(t);
        }
        // box of a warp and a sender: [column][lane]
        const uint32_t box = ring + static_cast<uint32_t>((warp - P16_FIRST_EPI) * SPLIT * OWN * 128 + lane * 4);
        __syncwarp();
        cluster_sync_all();                                  // every member's products are done: its ring is free
        if (ok) {
#pragma unroll
            for (int o = 0; o < SPLIT; ++o)
                if (o != member) {
                    const uint32_t to = map_to_cta(box + static_cast<uint32_t>(member * OWN * 128), static_cast<uint32_t>(o));
#pragma unroll
                    for (int c = 0; c < OWN; ++c) store_cluster(to + c * 128, acc[o * OWN + c]);
                }
        }
        __syncwarp();
        cluster_sync_all();
        if (ok) {
            float own[OWN], sum[OWN];
#pragma unroll
            for (int c = 0; c < OWN; ++c) {
                own[c] = acc[c];
#pragma unroll
                for (int o = 1; o < SPLIT; ++o) own[c] = o == member ? acc[o * OWN + c] : own[c];
                sum[c] = 0.0f;
            }
            const float *from = reinterpret_cast<const float *>(smem_raw + (box - raw));
#pragma unroll
            for (int o = 0; o < SPLIT; ++o)
#pragma unroll
                for (int c = 0; c < OWN; ++c) sum[c] += o == member ? own[c] : from[(o * OWN + c) * 32];
            P::template store<CG, BN>(p, t, sum, q * 32 + lane, part * R::COLS + member * OWN, staging);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (CG * SPLIT > 1) cluster_sync_all();   // no CTA leaves while another may still touch it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc<CG>(tmem_base, TMEM_COLUMNS);
    }
}

// Map over 16-bit elements [z][line][inner], box = 64 elements x box_lines lines, 128-byte swizzle, out-of-range elements read as zero.
// False where the driver does not take these strides.
inline bool make_map16(CUtensorMap *map, bool bf16, const void *base, int64_t inner, int64_t lines, int64_t ld, int64_t z, int64_t stride, int box_lines)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn || ld >= (1ll << 38) || stride >= (1ll << 38)) return false;
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(inner), static_cast<cuuint64_t>(lines), static_cast<cuuint64_t>(z)};
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(2 * ld), static_cast<cuuint64_t>(2 * stride)};
    cuuint32_t box[3] = {static_cast<cuuint32_t>(P16_BLOCK_K), static_cast<cuuint32_t>(box_lines), 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Matrices in plane pairs: [matrix][line][chunk of 64 elements][hi, lo][64], box = 64 elements of one plane x 64 lines
inline bool make_pair_map16(CUtensorMap *map, const void *base, int64_t chunks, int64_t lines, int64_t matrices)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(2 * chunks), static_cast<cuuint64_t>(lines), static_cast<cuuint64_t>(matrices)};
    cuuint64_t strides[3] = {128, static_cast<cuuint64_t>(256 * chunks), static_cast<cuuint64_t>(256 * chunks * lines)};
    cuuint32_t box[4] = {64, 1, 64, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class P, int CG, int BN, int PLANES, int SPLIT>
oz_status_t launch_product16(const typename P::Maps &maps, const typename P::Params &p, int64_t most_tiles, size_t table_bytes, cudaStream_t stream)
{
    auto kernel = product16_kernel<P, CG, BN, PLANES, SPLIT>;
    static std::atomic<unsigned long long> ready{0};
    // (one request for the largest table: the shared memory that a kernel may take is set once a device)
    OZ_CUDA_CHECK(allow_shared(kernel, kMaxShared, ready));
    // persistent CTAs; a cluster that shares its tile has one tile only
    int64_t groups = sm_count() / CG;
    if (SPLIT > 1 || most_tiles < groups) groups = most_tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(P16_THREADS);
    cfg.dynamicSmemBytes = P16_RING_BYTES + 1024 + P16_BARRIER_BYTES + table_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG * SPLIT;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    if (P::COOPERATIVE) {
        // blocks that wait for one another are on the device together: no more than it holds (asked once a device)
        static std::atomic<int> held[64];
        int dev = 0, most = 0;
        OZ_CUDA_CHECK(cudaGetDevice(&dev));
        most = held[dev & 63].load(std::memory_order_relaxed);
        if (most == 0) {
            cfg.gridDim = dim3(CG * SPLIT);
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            OZ_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&most, kernel, &cfg));
            if (most <= 0) return OZ_ERR_CUDA;
            held[dev & 63].store(most, std::memory_order_relaxed);
        }
        if (groups > most) groups = most;
        // an ordinary link in the stream, to both sides
        attr[1].id = cudaLaunchAttributeCooperative;
        attr[1].val.cooperative = 1;
    } else {
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
    }
    cfg.gridDim = dim3(static_cast<unsigned>(groups * CG * SPLIT));
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    OZ_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, maps, p));
    count_launch();
    return OZ_OK;
}

}  // namespace oz
