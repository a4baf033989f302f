// Losses at the output head for up to 16 tokens: the head streams by once per pass and every product is small beside it, so
// the operands go from memory straight into the registers of warp-level MMAs (m16n8k16), no tensor memory, no staging.
//
//   head_few_kernel<stats | grad>   z of 16 words at a time: the 16 warps of a CTA split K, add their parts in shared memory, and
//                                   a thread per word and token goes on with the maximum and sum it keeps (stats), or with
//                                   dz in bf16 (grad; T x N of them, a few MB)
//   head_few_grads_kernel           dW = dz^T x and dx = dz W from one more look at W, last words first: what the grad
//                                   kernel read last is still in the L2
//
// Rows of x that nothing is asked of enter as zeros.  Operands of both kernels are read as 16 bytes per lane: lane (g, t) =
// (lane / 4, lane % 4) takes columns 8 t .. 8 t + 7 of a block of 32 from rows g and g + 8.  Which column an MMA calls which
// index of its contraction is free as long as both operands agree, so the registers serve as they are; where the columns
// are not contracted over (dx, dW) `movmatrix` transposes registers as 8 x 8 tiles, whose columns then come out as 8 t + 2 j.
#pragma once

#include "head_words_tcgen05.cuh"

namespace sbn {

// What fits: the registers of a thread hold its share of the tokens' rows and of 16 words (and the same share of the next 16
// words under way), 80 of 128 registers for 16 tokens x 2560 or 96 for 8 tokens x 4096.
static inline bool head_few_takes(int T, int K) { return T <= 8 ? K <= 4096 : T <= 16 && K <= 2560; }
constexpr int kFewHeadWarps = 16;
constexpr int kFewHeadThreads = 32 * kFewHeadWarps;

// Up to this many entries per token every CTA sorts the targets itself (16 tokens x 65 entries: 130 comparisons per thread), which
// saves the launch of a kernel that takes 4 us; CTA 0 leaves them in memory for the kernels behind it.
constexpr int kFewOwnEvents = 65;

struct HeadFewParams {
    HeadTargets tg;
    HeadTargetsJob job;           // index null: the targets are in memory
    const uint16_t* x;            // [T][K]
    const uint16_t* w;            // [N][K]
    int T, N, K;
    float c0, inv_tau;
    float2* part;                 // stats: [T][parts], parts = CTAs
    float* part1;
    float* z_ev;                  // [T][events]
    const float *lse0, *lse1;
    HeadScale scale;
    uint16_t* dz;                 // grad: [T][ldz]
    int ldz;
    // gradients
    uint16_t* dw;                 // [N][K] or null
    float* acc;                   // [ranges][T][K] or null
    int slabs, per;               // 256-column slabs; blocks of 16 words per range
};

__device__ __forceinline__ void mma_bf16_k16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(b0));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint4 load_stream(const uint16_t* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// KBW: blocks of 32 columns per warp (K <= 512 KBW).  NT: groups of 8 tokens.  MODE, LIST, DUAL as in head_gemm_tcgen05.cuh.
template <int KBW, int NT, int MODE, bool LIST, bool DUAL>
__global__ void __launch_bounds__(kFewHeadThreads, 1)
head_few_kernel(const HeadFewParams p) {
    constexpr int kTok = 8 * NT;
    __shared__ float s_part[kFewHeadWarps][16][kTok];
    __shared__ int s_col[LIST ? kTok : 1][LIST ? kHeadMaxTop + 1 : 1];
    __shared__ float s_w[LIST ? kTok : 1][LIST ? kFewOwnEvents : 1];
    __shared__ int s_flags[kTok];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    const int blocks = (p.N + 15) >> 4, kbs = p.K >> 5;

    uint4 w[KBW][2];
    auto load_block = [&](int i, int nb) {
        const int kb = warp + kFewHeadWarps * i;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = nb * 16 + h * 8 + g;
            w[i][h] = make_uint4(0u, 0u, 0u, 0u);
            if (kb < kbs && nb < blocks && n < p.N) w[i][h] = load_stream(p.w + static_cast<size_t>(n) * p.K + kb * 32 + t4 * 8);
        }
    };
#pragma unroll
    for (int i = 0; i < KBW; ++i) load_block(i, blockIdx.x);

    const bool own = LIST && p.job.index != nullptr;
    if (own) {
        if (warp < p.T) {
            // (the room of the parts, which nobody has yet)
            int* col = reinterpret_cast<int*>(&s_part[0][0][0]) + warp * 2 * kFewOwnEvents;
            const int flags = warp_targets(p.job, warp, lane, col, reinterpret_cast<float*>(col + kFewOwnEvents), [&](int place, int c, float v) {
                s_col[LIST ? warp : 0][place] = c;
                s_w[LIST ? warp : 0][place] = v;
                if (blockIdx.x == 0) {
                    p.job.ev_col[warp * p.tg.events + place] = c;
                    p.job.ev_w[warp * p.tg.events + place] = v;
                }
            });
            if (lane == 0) {
                s_flags[warp] = flags;
                if (blockIdx.x == 0) {
                    p.job.flags[warp] = static_cast<unsigned char>(flags);
                    report_bad(flags);
                }
            }
        }
    } else if (tid < p.T) {
        s_flags[tid] = head_token_flags(p.tg, tid, p.N);
    }
    if (LIST && !own) {
        for (int i = tid; i < p.T * p.tg.events; i += kFewHeadThreads) s_col[i / p.tg.events][i % p.tg.events] = p.tg.ev_col[i];
    }
    __syncthreads();

    uint4 x[KBW][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = nt * 8 + g;
        const bool there = t < p.T && (s_flags[t] & (kRowDistill | kRowLabel));
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
            const int kb = warp + kFewHeadWarps * i;
            x[i][nt] = make_uint4(0u, 0u, 0u, 0u);
            if (there && kb < kbs) x[i][nt] = __ldg(reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(t) * p.K + kb * 32 + t4 * 8));
        }
    }
    // the word and token of this thread in every block
    const int tok = tid % kTok, slot = tid / kTok;
    const bool mine = slot < 16 && tok < p.T;
    const int flags = mine ? s_flags[tok] : 0;
    const bool asked = (flags & (kRowDistill | kRowLabel)) != 0;
    const int label = !LIST && asked ? static_cast<int>(p.tg.labels[tok]) : -1;
    constexpr float kLog2e = 1.4426950408889634f;
    float m = -INFINITY, s0 = 0.0f, s1 = 0.0f;
    float l0 = -INFINITY, l1 = -INFINITY, g0 = 0.0f, g1 = 0.0f;
    if constexpr (MODE == 1) {
        if (!LIST && blockIdx.x == 0 && mine) report_bad(flags);
        const float unit = head_scale_unit(warp_max(lane < p.T ? head_scale_share(p.scale, LIST, s_flags[lane], lane) : 0.0f));
        const float inv_scale = 1.0f / unit;
        if (blockIdx.x == 0 && tid == 0) p.scale.out[0] = unit;
        if (LIST ? (flags & kRowDistill) != 0 : asked) {
            l0 = -p.lse0[tok] * kLog2e;
            g0 = p.scale.g0[tok] * p.inv_tau * inv_scale;
        }
        if (DUAL && (flags & kRowLabel)) {
            l1 = -p.lse1[tok] * kLog2e;
            g1 = p.scale.g1[tok] * inv_scale;
        }
    }

    for (int nb = blockIdx.x; nb < blocks; nb += gridDim.x) {
        float d[NT][4] = {};
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                mma_bf16_k16(d[nt], w[i][0].x, w[i][1].x, w[i][0].y, w[i][1].y, x[i][nt].x, x[i][nt].y);
                mma_bf16_k16(d[nt], w[i][0].z, w[i][1].z, w[i][0].w, w[i][1].w, x[i][nt].z, x[i][nt].w);
            }
            load_block(i, nb + static_cast<int>(gridDim.x));          // the next block's words are under way during the rest
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            *reinterpret_cast<float2*>(&s_part[warp][g][nt * 8 + 2 * t4]) = make_float2(d[nt][0], d[nt][1]);
            *reinterpret_cast<float2*>(&s_part[warp][g + 8][nt * 8 + 2 * t4]) = make_float2(d[nt][2], d[nt][3]);
        }
        __syncthreads();
        const int n = nb * 16 + slot;
        if (mine) {
            float z = 0.0f;
#pragma unroll
            for (int v = 0; v < kFewHeadWarps; ++v) z += s_part[v][slot][tok];
            if (MODE == 0 && n < p.N && asked) {
                const float m_new = fmaxf(m, z);
                s0 = s0 * ex2_approx((m - m_new) * p.c0) + ex2_approx((z - m_new) * p.c0);
                if (DUAL) s1 = s1 * ex2_approx((m - m_new) * kLog2e) + ex2_approx((z - m_new) * kLog2e);
                m = m_new;
            }
            float v = 0.0f;
            if (MODE == 1 && n < p.N) {
                v = ex2_approx(fmaf(z, p.c0, l0)) * g0;
                if (DUAL) v = fmaf(ex2_approx(fmaf(z, kLog2e, l1)), g1, v);
            }
            if constexpr (LIST) {
                if (asked && n < p.N) {
                    int lo = 0, hi = p.tg.events;
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (s_col[tok][mid] < n) lo = mid + 1; else hi = mid;
                    }
                    for (; lo < p.tg.events && s_col[tok][lo] == n; ++lo) {
                        const size_t at = static_cast<size_t>(tok) * p.tg.events + lo;
                        if (MODE == 0) {
                            p.z_ev[at] = z;
                        } else {
                            const float q = own ? s_w[tok][lo] : p.tg.ev_w[at];
                            v -= q < 0.0f ? g1 : q * g0;
                        }
                    }
                }
            } else if (n == label) {
                if (MODE == 0) p.z_ev[tok] = z;
                else v -= g0;
            }
            if (MODE == 1) {
                unsigned short o;
                asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(o) : "f"(v));
                p.dz[static_cast<size_t>(tok) * p.ldz + n] = o;
            }
        }
        __syncthreads();
    }
    if constexpr (MODE == 0) {
        float* red = &s_part[0][0][0];                              // [3][16][kTok]
        if (slot < 16) {
            red[slot * kTok + tok] = m;
            red[(16 + slot) * kTok + tok] = s0;
            red[(32 + slot) * kTok + tok] = s1;
        }
        __syncthreads();
        if (tid < kTok && tid < p.T) {
            float mm = -INFINITY;
            for (int q = 0; q < 16; ++q) mm = fmaxf(mm, red[q * kTok + tid]);
            float a0 = 0.0f, a1 = 0.0f;
            for (int q = 0; q < 16; ++q) {
                const float mq = red[q * kTok + tid], sq = red[(16 + q) * kTok + tid];
                if (mq == -INFINITY && sq == 0.0f) continue;       // a slot without words
                a0 += sq * ex2_approx((mq - mm) * p.c0);
                if (DUAL) a1 += red[(32 + q) * kTok + tid] * ex2_approx((mq - mm) * kLog2e);
            }
            const size_t at = static_cast<size_t>(tid) * gridDim.x + blockIdx.x;
            p.part[at] = make_float2(mm, a0);
            if (DUAL) p.part1[at] = a1;
        }
    }
}

// CTA: 256 columns x a range of words.  Warp (column group of 64, part): blocks of 16 words part, part + 4, ... of the range.
template <int NT>
__global__ void __launch_bounds__(kFewHeadThreads, 1)
head_few_grads_kernel(const HeadFewParams p) {
    constexpr int kTok = 8 * NT, kDepth = 3;
    __shared__ float s_dx[256][kTok + 1];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int part = warp >> 2;
    const int slab = static_cast<int>(blockIdx.x) % p.slabs, range = static_cast<int>(blockIdx.x) / p.slabs;
    const int col0 = slab * 256 + (warp & 3) * 64;
    const bool live = col0 < p.K;                                   // K % 64 == 0: a group is in or out as a whole
    const int all = (p.N + 15) >> 4;
    const int first = range * p.per, last = min(all, first + p.per);

    // x^T as the B operand of dW: contraction over tokens, columns 8 t + 2 j of each block of 32
    uint32_t xt[2][4][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = nt * 8 + g;
        const bool there = live && t < p.T && (head_token_flags(p.tg, t, p.N) & (kRowDistill | kRowLabel));
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (there) v = __ldg(reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(t) * p.K + col0 + kb * 32 + t4 * 8));
            xt[kb][0][nt] = transpose_8x8(v.x);
            xt[kb][1][nt] = transpose_8x8(v.y);
            xt[kb][2][nt] = transpose_8x8(v.z);
            xt[kb][3][nt] = transpose_8x8(v.w);
        }
    }
    const float scale = p.scale.out[0];
    float acc[2][2][NT][4] = {};
    uint4 w[kDepth][2][2];
    uint32_t dz[kDepth][NT][2];
    // the range's blocks from its end: i-th of this warp
    auto block_at = [&](int i) { return last - 1 - part - 4 * i; };
    auto load = [&](int s, int nb) {
        const bool in = live && nb >= first;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = nb * 16 + h * 8 + g;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                w[s][kb][h] = make_uint4(0u, 0u, 0u, 0u);
                if (in && n < p.N && p.acc != nullptr) w[s][kb][h] = load_stream(p.w + static_cast<size_t>(n) * p.K + col0 + kb * 32 + t4 * 8);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int t = nt * 8 + g;
                dz[s][nt][h] = 0u;
                if (in && t < p.T) dz[s][nt][h] = __ldg(reinterpret_cast<const uint32_t*>(p.dz + static_cast<size_t>(t) * p.ldz + nb * 16 + h * 8 + 2 * t4));
            }
        }
    };
    const int mine = last - 1 - part < first ? 0 : (last - 1 - part - first) / 4 + 1;
#pragma unroll
    for (int s = 0; s < kDepth; ++s) load(s, block_at(s));
#pragma unroll 1
    for (int i = 0; i < mine; i += kDepth) {
#pragma unroll
        for (int s = 0; s < kDepth; ++s) {
            if (i + s >= mine) break;                               // the same for the whole warp
            const int nb = block_at(i + s);
            __syncwarp();
            if (p.acc != nullptr) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const uint32_t lo[4] = {w[s][kb][0].x, w[s][kb][0].y, w[s][kb][0].z, w[s][kb][0].w};
                    const uint32_t hi[4] = {w[s][kb][1].x, w[s][kb][1].y, w[s][kb][1].z, w[s][kb][1].w};
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t a0 = transpose_8x8(lo[2 * q]), a1 = transpose_8x8(lo[2 * q + 1]);
                        const uint32_t a2 = transpose_8x8(hi[2 * q]), a3 = transpose_8x8(hi[2 * q + 1]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_bf16_k16(acc[kb][q][nt], a0, a1, a2, a3, dz[s][nt][0], dz[s][nt][1]);
                    }
                }
            }
            if (p.dw != nullptr) {
                uint32_t a[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    a[nt][0] = transpose_8x8(dz[s][nt][0]);
                    a[nt][1] = transpose_8x8(dz[s][nt][1]);
                }
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    uint32_t o[2][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float d[4] = {};
                        if constexpr (NT == 1) mma_bf16_k8(d, a[0][0], a[0][1], xt[kb][j][0]);
                        else mma_bf16_k16(d, a[0][0], a[0][1], a[NT - 1][0], a[NT - 1][1], xt[kb][j][0], xt[kb][j][NT - 1]);
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[0][j]) : "f"(d[1] * scale), "f"(d[0] * scale));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[1][j]) : "f"(d[3] * scale), "f"(d[2] * scale));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int n = nb * 16 + h * 8 + g;
                        if (live && n < p.N)
                            *reinterpret_cast<uint4*>(p.dw + static_cast<size_t>(n) * p.K + col0 + kb * 32 + t4 * 8) = make_uint4(o[h][0], o[h][1], o[h][2], o[h][3]);
                    }
                }
            }
            load(s, block_at(i + s + kDepth));
        }
    }
    if (p.acc == nullptr) return;
    // the four parts one after another: a fixed order
#pragma unroll 1
    for (int turn = 0; turn < 4; ++turn) {
        if (part == turn) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // D row g or g + 8 = j 2 q or 2 q + 1, its column g / 2 * 8 + 2 j + g % 2 of the block; D column = token
                            const int c = (warp & 3) * 64 + kb * 32 + (g >> 1) * 8 + 2 * (2 * q + (e >> 1)) + (g & 1);
                            float& to = s_dx[c][nt * 8 + 2 * t4 + (e & 1)];
                            to = turn == 0 ? acc[kb][q][nt][e] : to + acc[kb][q][nt][e];
                        }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 256 * p.T; i += kFewHeadThreads) {
        const int c = i & 255, t = i >> 8;
        if (slab * 256 + c < p.K) p.acc[(static_cast<size_t>(range) * p.T + t) * p.K + slab * 256 + c] = s_dx[c][t];
    }
}

}  // namespace sbn
