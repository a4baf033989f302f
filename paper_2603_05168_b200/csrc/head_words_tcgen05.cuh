// The logits' tiles for up to 256 tokens: words on the lanes.  The head streams by once and is what such a call costs, so the
// tile is 128 words x all tokens on one CTA (`tcgen05.mma.cta_group::1`, M = 128, N = the tokens up to a multiple of 16): no row of the
// MMA is padding, every SM streams its own words, and a stage of 64 columns brings no more than the tokens there are.  With
// tokens on the lanes (head_gemm_tcgen05.cuh) 17 to 256 tokens cost the time of 256 rows per MMA: 2560 x 32000 took 46 to 60 us.
//
// The epilogue turns 32 words x 32 tokens at a time around through shared memory, so that a thread owns a token there too
// (HeadRow); a token's maximum and sums lie in shared memory between tiles, per warp.  Tokens that nothing is asked of stay where they are: their column of the product reaches nobody (stats) or is replaced
// by zeros (grad), and the grad kernel leaves a copy of x with zeros in their rows for dW.
//
//   warps       0 TMA producer, 1 MMA issuer (allocates TMEM), 2..5 epilogue: TMEM lane quarter w % 4
//   smem        stages of W 128 rows x 128 B | x rows x 128 B; 32 x 33 floats and 3 floats per token for each epilogue warp
//   TMEM        two accumulators of up to 256 columns, alternating
#pragma once

#include "head_gemm_tcgen05.cuh"

namespace sbn {

constexpr int kWordsTokens = 256;
constexpr int kWordsThreads = 192;
constexpr int kWordsTurnBytes = 4 * 32 * 33 * 4 + 512;                     // the four warps' squares, up to a multiple of 1 KB
constexpr int kWordsStateBytes = 4 * 3 * kWordsTokens * 4;                 // stats: [warp][m, s0, s1][token]; grad: the warps' boxes
static_assert(kWordsTurnBytes % 1024 == 0, "keeps the 1 KB alignment");

struct HeadWordsParams {
    HeadLogitsParams p;           // rows are tokens: count, row_src unused; parts = 4 x CTAs
    int tok_pad, stages;
    const uint16_t* x;            // grad: copied to xc [T up to a multiple of 64][K]
    uint16_t* xc;
    HeadScale scale;              // grad
};

static inline int words_stage_bytes(int tok_pad) { return 128 * 128 + tok_pad * 128; }
static inline int words_stages(int tok_pad) { return std::min(10, (232448 - kWordsTurnBytes - kWordsStateBytes - kBarrierBytes) / words_stage_bytes(tok_pad)); }
static inline int words_smem_bytes(int tok_pad) { return words_stages(tok_pad) * words_stage_bytes(tok_pad) + kWordsTurnBytes + kWordsStateBytes + kBarrierBytes; }

__device__ __forceinline__ void mma_bf16_one(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

template <int MODE, bool LIST, bool DUAL>
__global__ void __launch_bounds__(kWordsThreads, 1)
head_words_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadWordsParams wp) {
    const HeadLogitsParams& p = wp.p;
    pdl_launch_dependents();
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = smem_u32(smem_raw);
    if (smem_base & 1023u) {
        if (threadIdx.x == 0) atomicExch(&g_device_status, static_cast<int>(SBN_ERR_CUDA));
        return;
    }
    const int stages = wp.stages, stage_bytes = 128 * 128 + wp.tok_pad * 128;
    uint8_t* behind = smem_raw + stages * stage_bytes;
    float* turn = reinterpret_cast<float*>(behind);
    float* state = reinterpret_cast<float*>(behind + kWordsTurnBytes);
    const uint32_t bar_base = smem_base + stages * stage_bytes + kWordsTurnBytes + kWordsStateBytes;
    const uint32_t bar_full = bar_base, bar_empty = bar_full + 8 * stages;
    const uint32_t bar_acc_full = bar_empty + 8 * stages, bar_acc_empty = bar_acc_full + 16, tmem_slot = bar_acc_empty + 16;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + (tmem_slot + 8 - smem_base));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tiles = (p.v1 - p.v0 + 127) / 128, k_stages = p.K >> 6;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < stages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_acc_full + 8 * i, 1);
            mbar_init(bar_acc_empty + 8 * i, 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, kTmemCols);
        tcgen05_fence_before();
    }
    __syncthreads();
    tcgen05_fence_after();
    pdl_wait();
    uint32_t tmem_base;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot));

    if (warp == 0) {
        if (lane == 0 && !p.skip_loads) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = blockIdx.x; ok && i < tiles; i += gridDim.x) {
                for (int ks = 0; ks < k_stages; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    mbar_expect_tx(bar_full + 8 * stage, static_cast<uint32_t>(stage_bytes));
                    const uint32_t st = smem_base + stage * stage_bytes;
                    tma_load_2d(st, &maps.w, ks * 64, p.v0 + i * 128, bar_full + 8 * stage);
                    tma_load_2d(st + 128 * 128, &maps.x, ks * 64, 0, bar_full + 8 * stage);
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_idesc_bf16_any(128, wp.tok_pad, false, false);
            int stage = 0;
            uint32_t phase = 0, acc_iter = 0;
            bool ok = true;
            for (int i = blockIdx.x; ok && i < tiles; i += gridDim.x) {
                const uint32_t buf = acc_iter & 1u, acc_phase = (acc_iter >> 1) & 1u;
                if (!mbar_wait(bar_acc_empty + 8 * buf, acc_phase ^ 1u, abort_flag)) break;
                tcgen05_fence_after();
                for (int ks = 0; ks < k_stages; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                    const uint32_t st = smem_base + stage * stage_bytes;
                    const uint64_t a = make_smem_desc(st, 16, 1024, kSwz128), b = make_smem_desc(st + 128 * 128, 16, 1024, kSwz128);
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma_bf16_one(tmem_base + buf * 256u, a + 2 * q, b + 2 * q, idesc, (ks | q) != 0 ? 1u : 0u);
                    tcgen05_commit(bar_empty + 8 * stage);
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                tcgen05_commit(bar_acc_full + 8 * buf);
                ++acc_iter;
            }
        }
    } else {
        const int quarter = warp & 3;
        float* square = turn + quarter * (32 * 33);
        float* mine = state + quarter * 3 * kWordsTokens;
        const int all = MODE == 0 ? p.T : (p.T + 63) & ~63;                // grad: dW contracts over whole stages of 64 rows
        const int chunks = (all + 31) >> 5;
        const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
        HeadRow<MODE, LIST, DUAL> row;
        float inv_scale = 1.0f;
        const uint32_t box = smem_u32(state) + static_cast<uint32_t>(quarter * kWarpBoxBytes);       // grad: no state
        if constexpr (MODE == 0) {
            for (int c = 0; c < chunks; ++c) {
                mine[c * 32 + lane] = -INFINITY;
                mine[kWordsTokens + c * 32 + lane] = 0.0f;
                mine[2 * kWordsTokens + c * 32 + lane] = 0.0f;
            }
        } else {
            float largest = 0.0f;                                          // every warp for itself
            for (int t = lane; t < p.T; t += 32) largest = fmaxf(largest, head_scale_share(wp.scale, p.tg, t, p.N));
            const float unit = head_scale_unit(warp_max(largest));
            inv_scale = 1.0f / unit;
            if (blockIdx.x == 0 && threadIdx.x == 64) {
                wp.scale.out[0] = unit;
                wp.scale.out[1] = inv_scale;
            }
            // x for dW, zeros in rows that nothing is asked of and behind the last token
            const int vecs = p.K >> 3;
            for (int t = blockIdx.x; t < all; t += gridDim.x) {
                const int flags = t < p.T ? head_token_flags(p.tg, t, p.N) : 0;
                const bool there = (flags & (kRowDistill | kRowLabel)) != 0;
                if (!LIST && threadIdx.x == 64) report_bad(flags);
                const uint4* from = reinterpret_cast<const uint4*>(wp.x + static_cast<size_t>(t) * p.K);
                uint4* to = reinterpret_cast<uint4*>(wp.xc + static_cast<size_t>(t) * p.K);
                for (int v = threadIdx.x - 64; v < vecs; v += 128) to[v] = there ? __ldg(from + v) : make_uint4(0u, 0u, 0u, 0u);
            }
        }
        uint32_t acc_iter = 0;
        for (int i = blockIdx.x; i < tiles; i += gridDim.x) {
            const uint32_t buf = acc_iter & 1u, acc_phase = (acc_iter >> 1) & 1u;
            const int n0 = p.v0 + i * 128 + quarter * 32;
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_acc_full + 8 * buf, acc_phase, abort_flag))) break;
            tcgen05_fence_after();
            const uint32_t t_addr = tmem_base + lane_base + buf * 256u;
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                uint32_t z[32];
                __syncwarp();
                tmem_ld_32x32b_x32(t_addr + static_cast<uint32_t>(c * 32), z);
                tmem_ld_wait();
                if (c + 1 == chunks) {
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_acc_empty + 8 * buf);
                }
#pragma unroll
                for (int q = 0; q < 32; ++q) square[q * 33 + lane] = __uint_as_float(z[q]);
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 32; ++q) z[q] = __float_as_uint(square[lane * 33 + q]);
                const int t = c * 32 + lane;
                const bool here = t < p.T && (head_token_flags(p.tg, t, p.N) & (kRowDistill | kRowLabel));
                row.begin(p, t, here ? t : 0, here, inv_scale);
                row.seek(p, n0);
                if constexpr (MODE == 0) {
                    row.m = mine[t];
                    row.s0 = mine[kWordsTokens + t];
                    if (DUAL) row.s1 = mine[2 * kWordsTokens + t];
                    row.note_targets(p, n0, [&](int q) { return square[lane * 33 + q]; });
                    row.stats(p, z, n0);
                    __syncwarp();
                    mine[t] = row.m;
                    mine[kWordsTokens + t] = row.s0;
                    if (DUAL) mine[2 * kWordsTokens + t] = row.s1;
                } else {
                    uint32_t o[16];
                    row.grad(p, z, n0, o);
                    store_warp_box(box, lane, o, [&] { tma_store_2d(&maps.dz, n0 - p.v0, c * 32, box); });
                }
            }
            ++acc_iter;
        }
        if constexpr (MODE == 1) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        } else {
            for (int c = 0; c < chunks; ++c) {
                const int t = c * 32 + lane;
                if (t >= p.T) break;
                row.begin(p, t, t, true);
                row.m = mine[t];
                row.s0 = mine[kWordsTokens + t];
                if (DUAL) row.s1 = mine[2 * kWordsTokens + t];
                row.store_part(p, static_cast<int>(blockIdx.x) * 4 + quarter);
            }
        }
    }

    tcgen05_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

}  // namespace sbn
