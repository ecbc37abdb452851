// um_pair_gemm.cuh -- D = A B^T on pairs of SMs (tcgen05.mma.cta_group::2), bf16
// operands, fp32 accumulators: a persistent kernel with 256 x n_tile output
// tiles and an epilogue of the caller's.
//
// A cluster of two CTAs makes a tile: each holds 128 rows of A and half of the
// tile's columns of B in shared memory, and the accumulators of its 128 rows
// in its own TMEM.  One k block of 64 is 16 KiB of A and up to 16 KiB of B a
// CTA, half of B's bytes of a one-CTA tile of the same shape; that is what
// the pair is for, because a 128 x 256 tile on one SM would read 96 bytes a
// cycle from shared memory and take as many by copies.  Two accumulators of
// up to 256 columns fill TMEM, so that the epilogue of a tile runs under the
// products of the next one.
//
// Each operand is K-major (rows of A or B, k contiguous) or MN-major (rows of
// k, the row index of A or B contiguous), so that a matrix and its transpose
// are read from the same memory.
//
// The tensor cores cut off what a sum loses in its last place, so a sum of many
// steps of 16 k comes out short: logits of 2048 k by 1e-6 of their size.  That is
// far below a rounding to bf16 but not below fp32.  An operation with kSumBlocks
// ends the sum in the tensor cores after so many k blocks; the epilogue adds it
// to the tile's (rounded to nearest), which it holds in registers, while the
// products go on in the other accumulator.  (Held so for every operation, the
// products were 2 to 4 % slower.)
//
// EXACT: operands of fp32 values, each three bf16 planes that add up to it.  A
// k block's three planes of A and of B are copied once and multiplied in
// the six pairs that reach 2^-24 of the product, the smallest first, a sum a k
// block (24 steps).  (Gradient of 333 tokens against 5003 x 509: relative error
// 3e-6 with one sum a tile, 4e-7 so; 146 us with each pair of planes copied for
// itself, 111 so.)
//
// Warps of a CTA: 0 copies (TMA, one elected thread), 1 products (one thread
// of the pair's first CTA), 2-9 epilogue (four for each half of the columns: with
// four in all, tiles of up to 16 k blocks took as long as their epilogue).  Waits are
// bounded; one that gives up sets the error word, and the others run into their own
// limits.
#pragma once

#include "um_internal.cuh"
#include "um_tc.cuh"

namespace um {
namespace pair {

constexpr int kEpilogue = 8;                             // warps
constexpr int kThreads = (2 + kEpilogue) * 32;
constexpr int kTileM = 256;
constexpr uint32_t kOperand = 128 * 128;                  // 128 rows (or columns) x 64 k
constexpr uint32_t kGroupBytes = 64 * 128;                // MN-major: 64 columns x 64 k

// Shared memory of an epilogue warp, to turn rows by threads into rows by
// lanes (an odd row: no bank conflicts either way).
template <int COLS> struct Scratch {
    static constexpr int kCols = COLS;
    float v[32][COLS + 1];
};

template <bool EXACT> struct Shape {
    static constexpr int kMaxN = EXACT ? 128 : 256;
    static constexpr int kPlanes = EXACT ? 3 : 1;
    static constexpr int kStages = EXACT ? 3 : 6;
    static constexpr uint32_t kB = kOperand * kMaxN / 256;        // a CTA's half of the columns
    static constexpr uint32_t kStage = kPlanes * (kOperand + kB);
    using Turn = Scratch<EXACT ? 8 : 16>;                         // what fits
    static constexpr size_t kSmem = (size_t)kStages * kStage + 1024 + kEpilogue * sizeof(Turn);
};

struct Plan {
    int m_tiles, n_tiles, n_tile, splits;    // splits: of the k blocks, a tile each
    int k_blocks;
    int group_m;                             // row tiles that run side by side
    int *err;
};

struct Tile {
    int m0, n0, split, kb0, kb1;             // first row and column, k blocks [kb0, kb1)
    __device__ __forceinline__ Tile(const Plan &p, int item) {
        const int tiles = p.m_tiles * p.n_tiles;
        split = item / tiles;
        int i = item - split * tiles;
        const int band = p.group_m * p.n_tiles, g = i / band;
        i -= g * band;
        const int height = min(p.group_m, p.m_tiles - g * p.group_m);
        n0 = i / height * p.n_tile;
        m0 = (g * p.group_m + i % height) * kTileM;
        kb0 = 0;
        kb1 = p.k_blocks;
        if (p.splits > 1) {                  // splits <= 64, k_blocks < 2^24
            kb0 = (int)((uint32_t)p.k_blocks * (uint32_t)split / (uint32_t)p.splits);
            kb1 = (int)((uint32_t)p.k_blocks * (uint32_t)(split + 1) / (uint32_t)p.splits);
        }
    }
};

// ---- what differs from one CTA's instructions ---------------------------------

// a copy whose bytes are counted by a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load(void *dst, const CUtensorMap *map, uint32_t bar, int x,
                                         int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(tc::smem_u32(dst)),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}
// Relaxed: what it tells of are loads from TMEM, which tcgen05's fence orders; a
// release for the cluster would also wait until the epilogue's stores are in L2.
__device__ __forceinline__ void remote_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
}
__device__ __forceinline__ bool wait_cluster(uint64_t *bar, uint32_t parity) {
    const long long start = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(tc::smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - start > tc::kWaitLimitCycles) return false;
    }
}
__device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                    uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// arrives on `bar` of both CTAs once this thread's products so far are done
__device__ __forceinline__ void commit_both(uint64_t *bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(tc::smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *dst, uint32_t ncols) {   // whole warp
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     tc::smem_u32(dst)),
                 "r"(ncols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {   // whole warp
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
}

// 32 columns of this thread's accumulator row
__device__ __forceinline__ void load32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    __syncwarp();                            // an operation may leave lanes early
    tc::tmem_ld32_nowait(taddr, r);
    tc::tmem_ld_wait();
    tc::arrived(r);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// A thread's sums of its row, 32 columns at a time, to be used up: in registers, or
// (C = 0) read from TMEM into the place given as they are asked for.
template <int C> struct Sums {
    static constexpr int kChunks = C;
    float v[C][32];
    using Chunk = float (&)[32];
    __device__ __forceinline__ Chunk get(int i, float (&)[32]) { return v[i]; }
};
template <> struct Sums<0> {
    static constexpr int kChunks = 4;
    uint32_t tmem;
    using Chunk = float (&)[32];
    __device__ __forceinline__ Chunk get(int i, float (&z)[32]) {
        load32(tmem + 32 * i, z);
        return z;
    }
};

// Epi: epi(tile, row, sums, half, c0, c1, fetched, scratch) by the threads of the
// epilogue: the tile's row (0..255) of this thread, its sums of columns [c0, c1)
// (c0 a multiple of 32) in 32s, which half of the columns that is, what
// fetch(tile, row) loaded while the tile before was worked on, and the warp's scratch.
// Epi::kSumBlocks: k blocks of a sum in the tensor cores, 0 for all of a tile.
template <class Epi, bool A_MN, bool B_MN, bool EXACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap map_a,
                const __grid_constant__ CUtensorMap map_b, Plan p, Epi epi) {
    using S = Shape<EXACT>;
    constexpr int kStages = S::kStages;
    constexpr int kSum = EXACT ? 1 : Epi::kSumBlocks;    // k blocks of a sum
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_base;
    uint8_t *ring = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_ctarank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&full[s], 1);      // the first CTA's counts both CTAs' copies
            tc::mbar_init(&empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&acc_full[i], 1);
            tc::mbar_init(&acc_empty[i], 2 * kEpilogue);   // the warps of both CTAs
        }
        tc::mbar_init(&drained, 1);
        tc::fence_mbar_init();
        tc::prefetch_tensormap(&map_a);
        tc::prefetch_tensormap(&map_b);
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    if (w == 1) tmem_alloc(&tmem_base, 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();                      // the peer's barriers and TMEM are there
    tc::tc_fence_after();
    const uint32_t tmem = tmem_base;
    const int items = p.m_tiles * p.n_tiles * p.splits;
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
    bool ok = true;

    if (w == 0) {
        if (lane == 0) {
            const uint32_t half = (uint32_t)p.n_tile / 2;
            const uint32_t bytes = 2 * S::kPlanes * (kOperand + half * 128);
            int s = 0, issued = 0;
            uint32_t phase = 0;
            for (int item = first; ok && item < items; item += step) {
                const Tile t(p, item);
                const int m0 = t.m0 + 128 * (int)rank, n0 = t.n0 + (int)(half * rank);
                for (int kb = t.kb0; kb < t.kb1; ++kb) {
                    if (!(ok = wait_cluster(&empty[s], phase ^ 1))) break;
                    if (rank == 0) tc::mbar_arrive_expect_tx(&full[s], bytes);
                    const uint32_t bar = tc::mapa_shared(tc::smem_u32(&full[s]), 0);
                    uint8_t *at = ring + (size_t)s * S::kStage;
#pragma unroll
                    for (int z = 0; z < S::kPlanes; ++z) {
                        uint8_t *a = at + z * kOperand;
                        uint8_t *b = at + S::kPlanes * kOperand + z * S::kB;
                        if (A_MN) {
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                tma_load(a + j * kGroupBytes, &map_a, bar, m0 + 64 * j, kb * 64, z);
                        } else {
                            tma_load(a, &map_a, bar, kb * 64, m0, z);
                        }
                        if (B_MN) {
                            for (uint32_t j = 0; j < half / 64; ++j)
                                tma_load(b + j * kGroupBytes, &map_b, bar, n0 + 64 * (int)j,
                                         kb * 64, z);
                        } else {
                            tma_load(b, &map_b, bar, kb * 64, n0, z);
                        }
                    }
                    ++issued;
                    if (++s == kStages) {
                        s = 0;
                        phase ^= 1;
                    }
                }
            }
            // the last products' arrivals at this CTA's barriers, before it may leave
            for (int i = 0; ok && i < kStages && i < issued; ++i) {
                if (--s < 0) {
                    s = kStages - 1;
                    phase ^= 1;
                }
                ok = wait_cluster(&empty[s], phase);
            }
            if (!ok) {
                atomicOr(p.err, kErrTimeout);
                // copies in flight end by themselves: give them far longer than they take
                const long long start = clock64();
                while (clock64() - start < 4000000ll) __nanosleep(1000);
            }
        }
    } else if (w == 1) {
        if (rank == 0 && lane == 0) {
            const uint32_t idesc = tc::idesc_bf16_f32(kTileM, 0) | ((uint32_t)(p.n_tile >> 3) << 17) |
                                   (A_MN ? tc::kAColumns : 0u) |
                                   (B_MN ? tc::kBColumns : 0u);
            const uint32_t base = tc::smem_u32(ring);
            const uint64_t a_desc = A_MN ? tc::desc_mn_sw128(base, kGroupBytes) : tc::desc_k_sw128(base);
            constexpr uint32_t b_at = S::kPlanes * kOperand;
            const uint64_t b_desc = B_MN ? tc::desc_mn_sw128(base + b_at, kGroupBytes)
                                         : tc::desc_k_sw128(base + b_at);
            // 16 k further: 16 rows of 128 bytes (MN-major), or 32 bytes along the rows
            constexpr uint32_t a_step = (A_MN ? 16 * 128 : 32) >> 4;
            constexpr uint32_t b_step = (B_MN ? 16 * 128 : 32) >> 4;
            int s = 0;
            uint32_t phase = 0, n = 0;
            for (int item = first; ok && item < items; item += step) {
                const Tile t(p, item);
                const int blocks = t.kb1 - t.kb0, most = kSum ? kSum : blocks;
                for (int b0 = 0; ok && b0 < blocks; b0 += most, ++n) {
                    const int buf = n & 1;
                    if (!(ok = wait_cluster(&acc_empty[buf], ((n >> 1) & 1) ^ 1))) break;
                    tc::tc_fence_after();
                    const uint32_t d = tmem + buf * S::kMaxN;
                    for (int kb = b0; kb < min(blocks, b0 + most); ++kb) {
                        if (!(ok = wait_cluster(&full[s], phase))) break;
                        tc::tc_fence_after();
                        const uint32_t at = (uint32_t)s * (S::kStage >> 4);
#pragma unroll
                        for (int i = 0; i < (EXACT ? 6 : 1); ++i) {
                            // pairs of planes: the smallest products first
                            constexpr int plane_a[6] = {2, 1, 0, 1, 0, 0};
                            constexpr int plane_b[6] = {0, 1, 2, 0, 1, 0};
                            const uint32_t pa = EXACT ? plane_a[i] * (kOperand >> 4) : 0;
                            const uint32_t pb = EXACT ? plane_b[i] * (S::kB >> 4) : 0;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma(d, a_desc + at + pa + k * a_step, b_desc + at + pb + k * b_step,
                                    idesc, kb > b0 || i > 0 || k > 0);
                        }
                        commit_both(&empty[s]);
                        if (++s == kStages) {
                            s = 0;
                            phase ^= 1;
                        }
                    }
                    if (ok) commit_both(&acc_full[buf]);
                }
            }
            if (!ok) {       // products in flight end before anything is freed
                atomicOr(p.err, kErrTimeout);
                asm volatile(
                    "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                        tc::smem_u32(&drained))
                    : "memory");
                tc::mbar_wait(&drained, 0);
            }
        }
    } else {
        const int quarter = w & 3;
        const int row = 128 * (int)rank + quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        typename S::Turn &scratch =
            reinterpret_cast<typename S::Turn *>(ring + (size_t)kStages * S::kStage)[w - 2];
        const int half = (w - 2) >> 2, middle = (p.n_tile / 2 + 31) & ~31;
        const int c0 = half ? middle : 0, c1 = half ? p.n_tile : middle;
        uint32_t n = 0;
        Tile t(p, first);
        auto fetched = epi.fetch(t, row);
        for (int item = first; ok && item < items; item += step) {
            const int sums = kSum ? (t.kb1 - t.kb0 + kSum - 1) / kSum : 1;
            Sums<kSum ? S::kMaxN / 64 : 0> all;
            const Tile next(p, item + step < items ? item + step : item);
            const auto ahead = epi.fetch(next, row);
            for (int i = 0; i < sums; ++i, ++n) {
                const int buf = n & 1;
                ok = __all_sync(0xffffffffu, wait_cluster(&acc_full[buf], (n >> 1) & 1));
                if (!ok) break;
                tc::tc_fence_after();
                const uint32_t at = lanes + buf * S::kMaxN + c0;
                if constexpr (kSum == 0) {
                    all.tmem = at;
                    epi(t, row, all, half, c0, c1, fetched, scratch);
                } else {
#pragma unroll
                    for (int c = 0; c < S::kMaxN / 64; ++c) {
                        if (c0 + 32 * c >= c1) break;
                        if (i == 0) {
                            load32(at + 32 * c, all.v[c]);
                        } else {
                            float x[32];
                            load32(at + 32 * c, x);
#pragma unroll
                            for (int k = 0; k < 32; ++k) all.v[c][k] += x[k];
                        }
                    }
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) remote_arrive(tc::mapa_shared(tc::smem_u32(&acc_empty[buf]), 0));
            }
            if constexpr (kSum != 0)
                if (ok) epi(t, row, all, half, c0, c1, fetched, scratch);
            t = next;
            fetched = ahead;
        }
        if (!ok && lane == 0) atomicOr(p.err, kErrTimeout);
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();                      // nothing of the peer's is in use any more
    tc::tc_fence_after();
    if (w == 1) tmem_dealloc(tmem, 512);
}

}  // namespace pair
}  // namespace um
