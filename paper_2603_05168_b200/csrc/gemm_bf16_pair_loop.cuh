// The main loop of a bf16 GEMM on CTA pairs, for kernels that differ in what they multiply and in what becomes of the
// accumulators (the output head's logits and gradients, head_gemm_tcgen05.cuh).  Two CTAs of a cluster issue one
// `tcgen05.mma.cta_group::2.kind::f16` (M = 256: each CTA supplies 128 rows of A and half of a B tile and keeps its 128 x 256
// slice of the accumulator in its own tensor memory); TMA fills stages of 64 contraction steps.  No TMA multicast.  All
// waits are bounded.  Two shapes of tiles:
//
//   narrow  256 x BN, BN <= 256.  The two 256-column halves of tensor memory alternate as accumulators, so the epilogue of a tile
//           runs under the next tile's MMAs.  Per CTA and stage A 16 KB | B BN/2 rows x 128 B (<= 16 KB), 6 or 7 stages
//   wide    256 x 512.  Both halves are one tile's: a stage of A serves two MMAs, so the loop brings 24 KB per 256 x 256 x 64 into an
//           SM instead of 32.  With narrow tiles 148 SMs take 11 TB/s from the L2, which is what it gives (0.41 us per stage
//           where the MMAs need 0.27 at full clock), and every byte costs power that the MMAs need.  The next tile's MMAs wait
//           until the epilogue has read the accumulators out: 16 warps instead of 8.  A 16 KB | B 32 KB, 4 stages.
//           CTA r loads B rows (columns of the tile) 256 r .. 256 r + 255 as one box; MMA h takes 128 of them from each CTA, so
//           accumulator h holds the tile's columns 128 h .. and 256 + 128 h ..; a half tile (256 columns) uses accumulator 0 alone
//
//   warps        0 TMA producer (both CTAs), 1 MMA issuer (leader CTA only; both allocate TMEM),
//                2.. epilogue: warp w reads TMEM lane quarter w % 4; its `sub` = (w - 2) / 4 says which columns (narrow: even or odd
//                chunks of 32; wide: accumulator sub / 2, columns 128 (sub % 2) .., that is 128 (sub / 2) + 256 (sub % 2) .. of the tile)
//
// A `Work` has the kernel's parameters and gives
//   kWide, kStages, kStagingBytes  shape, stages of kStageBytes, and shared memory behind them for the epilogue
//   stages(), stage_bytes()        the same, or more and smaller stages where a tile has few columns
//   start()                        what it reads from memory for itself, after the dependency wait
//   Tile                           a tile: at least { int k_stages; int bn; }
//   Tiles(work, pair)              the tiles of a CTA pair in order: bool next(Tile&)
//   load(tile, ks, rank, st, bar)  issues stage ks of the tile for this CTA: A at st, B at st + kPairLoopStageA
//   idesc(tile), a_desc(tile, st), a_step(tile), b_desc(tile, st), b_step(tile)   operand descriptors and their advance per MMA
//   Epilogue(work, rank, quarter, sub, lane, staging): begin(tile) before the accumulator is there, then
//                                  run(tile, taddr, release); finish() after the last tile
// All epilogue warps of a CTA take a narrow tile or none does (a barrier with a vote): its epilogue may synchronise its warps.
#pragma once

#include "gemm_bf16_pair_tcgen05.cuh"

namespace sbn {

constexpr int kPairLoopStageA = 128 * 128;                    // bytes
constexpr int kPairLoopStageB = 128 * 128;                    // bytes of one MMA's half of B
template <class Work>
struct PairLoop {
    static constexpr int kEpiWarps = Work::kWide ? 16 : 8;
    static constexpr int kThreads = 32 * (2 + kEpiWarps);
    static constexpr int kStageBytes = kPairLoopStageA + (Work::kWide ? 2 : 1) * kPairLoopStageB;
    static constexpr int kSmemBytes = Work::kStages * kStageBytes + Work::kStagingBytes + kBarrierBytes;
    static_assert(kSmemBytes <= 232448 && Work::kStagingBytes % 1024 == 0, "shared memory overflow");
};

// Whether all epilogue warps of a CTA say yes (narrow tiles).
__device__ __forceinline__ bool epilogue_all(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"(static_cast<uint32_t>(ok)) : "memory");
    return all != 0;
}

// Instruction descriptor for kind::f16: D = fp32, A = B = bf16; either operand K-major or MN-major.
__host__ __device__ constexpr uint32_t make_idesc_bf16_any(int mma_m, int mma_n, bool a_mn_major, bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (a_mn_major ? (1u << 15) : 0u) | (b_mn_major ? (1u << 16) : 0u) |
           (static_cast<uint32_t>(mma_n >> 3) << 17) | (static_cast<uint32_t>(mma_m >> 4) << 24);
}

template <class Work>
__device__ __forceinline__ void bf16_pair_loop(Work& work, const bool skip_loads) {
    constexpr int EPI_WARPS = PairLoop<Work>::kEpiWarps;
    const int STAGES = work.stages(), STAGE_BYTES = work.stage_bytes();
    constexpr bool WIDE = Work::kWide;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = smem_u32(smem_raw);
    if (smem_base & 1023u) {          // swizzled tiles need 1 KB alignment; identical in every CTA
        if (threadIdx.x == 0) atomicExch(&g_device_status, static_cast<int>(SBN_ERR_CUDA));
        return;
    }
    const uint32_t staging = smem_base + static_cast<uint32_t>(STAGES * STAGE_BYTES);
    const uint32_t bar_full = staging + Work::kStagingBytes;
    const uint32_t bar_empty = bar_full + 8 * STAGES;
    const uint32_t bar_acc_full = bar_empty + 8 * STAGES;     // [2]
    const uint32_t bar_acc_empty = bar_acc_full + 16;         // [2]
    const uint32_t tmem_slot = bar_acc_empty + 16;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + (tmem_slot + 8 - smem_base));

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair_id = blockIdx.x >> 1;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_acc_full + 8 * i, 1);
            mbar_init(bar_acc_empty + 8 * i, 2 * EPI_WARPS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, kTmemCols);
        tcgen05_fence_before();
    }
    __syncthreads();
    cluster_sync_all();
    tcgen05_fence_after();
    pdl_wait();                       // nothing above touches global memory
    work.start();
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0 && !skip_loads) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            typename Work::Tiles tiles(work, pair_id);
            typename Work::Tile t;
            while (ok && tiles.next(t)) {
                const uint32_t bytes_per_cta = static_cast<uint32_t>(kPairLoopStageA + (t.bn >> 1) * 128);
                for (int ks = 0; ks < t.k_stages; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t full_leader = map_to_cta(bar_full + 8 * stage, 0);
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * stage, 2 * bytes_per_cta);
                    // rows or columns beyond the tensors are zero-filled by the hardware and still count their full size
                    work.load(t, ks, rank, smem_base + static_cast<uint32_t>(stage * STAGE_BYTES), full_leader);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (leader)
        if (rank == 0 && lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            uint32_t acc_iter = 0;
            bool ok = true;
            typename Work::Tiles tiles(work, pair_id);
            typename Work::Tile t;
            while (ok && tiles.next(t)) {
                const uint32_t idesc = work.idesc(t);
                const uint64_t a_step = work.a_step(t), b_step = work.b_step(t);
                const uint32_t buf = WIDE ? 0u : acc_iter & 1u;
                const uint32_t acc_phase = (WIDE ? acc_iter : acc_iter >> 1) & 1u;
                if (!mbar_wait(bar_acc_empty + 8 * buf, acc_phase ^ 1u, abort_flag)) break;
                tcgen05_fence_after();
                const uint32_t d_tmem = tmem_base + buf * 256u;
                for (int ks = 0; ks < t.k_stages; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                    const uint32_t st = smem_base + static_cast<uint32_t>(stage * STAGE_BYTES);
                    const uint64_t a_desc = work.a_desc(t, st), b_desc = work.b_desc(t, st + kPairLoopStageA);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        mma_bf16_pair(d_tmem, a_desc + a_step * q, b_desc + b_step * q, idesc, (ks | q) != 0 ? 1u : 0u);
                        if (WIDE && t.bn == 512)
                            mma_bf16_pair(d_tmem + 256u, a_desc + a_step * q, b_desc + (kPairLoopStageB >> 4) + b_step * q, idesc, (ks | q) != 0 ? 1u : 0u);
                    }
                    tcgen05_commit_pair(bar_empty + 8 * stage);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                tcgen05_commit_pair(bar_acc_full + 8 * buf);
                ++acc_iter;
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        const int quarter = warp & 3;                     // TMEM lane quarter this warp may read
        const int sub = (warp - 2) >> 2;
        const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
        uint32_t acc_iter = 0;
        typename Work::Tiles tiles(work, pair_id);
        typename Work::Tile t;
        typename Work::Epilogue epi(work, static_cast<int>(rank), quarter, sub, lane, staging);
        while (tiles.next(t)) {
            const uint32_t buf = WIDE ? 0u : acc_iter & 1u;
            const uint32_t acc_phase = (WIDE ? acc_iter : acc_iter >> 1) & 1u;
            const uint32_t acc_empty_leader = map_to_cta(bar_acc_empty + 8 * buf, 0);
            epi.begin(t);
            const bool there = mbar_wait(bar_acc_full + 8 * buf, acc_phase, abort_flag);
            if (WIDE ? !__all_sync(0xFFFFFFFFu, there) : !epilogue_all(there)) break;
            tcgen05_fence_after();
            // gives the accumulator back; once per tile and warp, after the warp's last read of it
            auto release = [&] {
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc_empty_leader);
            };
            epi.run(t, tmem_base + lane_base + buf * 256u, release);
            ++acc_iter;
        }
        epi.finish();
    }

    // teardown: nobody leaves while the peer may still touch this CTA's smem, barriers or TMEM
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

}  // namespace sbn
