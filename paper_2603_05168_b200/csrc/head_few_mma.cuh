// Losses at the output head for up to 16 tokens: the head streams by once per pass and every product is small beside it, so
// the operands go from memory straight into the registers of warp-level MMAs, no tensor memory, no staging of words.
//
//   head_few_forward_kernel    z of 16 words at a time: the 16 warps of a CTA split K, add their parts in shared memory, and a thread per
//                              word and token goes on with the maximum and sum it keeps
//   head_few_backward_kernel   8 words at a time, everything from one look at them: z as above, dz in bf16 in shared memory, then
//                              every warp forms dW's rows of its columns and adds to its columns of dx, which it keeps in
//                              registers for the whole kernel (one partial sum per CTA for head_dx_kernel).  With dz kept in
//                              memory and the words read a second time for dx, 7 tokens x 3968 x 139152 took 630 us
//
// Rows of x that nothing is asked of enter as zeros.  Operands are read as 16 bytes per lane: lane (g, t) = (lane / 4, lane % 4)
// takes columns 8 t .. 8 t + 7 of a block of 32 from row g (and g + 8).  Which column an MMA calls which index of its contraction
// is free as long as both operands agree, so the registers serve as they are; where the columns are not contracted over (dx,
// dW) `movmatrix` transposes registers as 8 x 8 tiles, whose columns then come out as 8 t + 2 j.
#pragma once

#include "head_words_tcgen05.cuh"

namespace sbn {

// What fits the 128 registers of a thread: forward its share of the tokens' rows and of 16 words, 80 for 16 tokens x 2560 or 96
// for 8 tokens x 4096; backward its share of dx and of 8 words, 100 and 96.
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
    float c0, c1, inv_tau;        // log2(e) / tau and log2(e), times head_logit_scale
    float2* part;                 // stats: [T][parts], parts = CTAs
    float* part1;
    float* z_ev;                  // [T][events]
    const float *lse0, *lse1;
    HeadScale scale;
    uint16_t* dw;                 // [N][K] or null
    float* acc;                   // [CTAs][T][K] or null
};

__device__ __forceinline__ void mma_bf16_k16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

// What is asked of the tokens, for a CTA: flags, and the sorted targets of a distillation.
template <int NT, bool LIST>
struct FewTargets {
    int flags[8 * NT];
    int col[LIST ? 8 * NT : 1][LIST ? kHeadMaxTop + 1 : 1];
    float w[LIST ? 8 * NT : 1][LIST ? kFewOwnEvents : 1];
};
// `room`: 2 kFewOwnEvents words per token, free until the barrier that the caller puts behind this.
template <int NT, bool LIST>
__device__ __forceinline__ void few_targets(const HeadFewParams& p, FewTargets<NT, LIST>& s, int* room) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (LIST && p.job.index != nullptr) {
        if (warp < p.T) {
            int* col = room + warp * 2 * kFewOwnEvents;
            int heaviest;
            const int flags = warp_targets(p.job, warp, lane, col, reinterpret_cast<float*>(col + kFewOwnEvents), &heaviest, [&](int place, int c, float v) {
                s.col[LIST ? warp : 0][place] = c;
                s.w[LIST ? warp : 0][place] = v;
                if (blockIdx.x == 0) {
                    p.job.ev_col[warp * p.tg.events + place] = c;
                    p.job.ev_w[warp * p.tg.events + place] = v;
                }
            });
            if (lane == 0) {
                s.flags[warp] = flags;
                if (blockIdx.x == 0) {
                    p.job.flags[warp] = static_cast<unsigned char>(flags);
                    p.job.ev_top[warp] = heaviest;
                    report_bad(flags);
                }
            }
        }
    } else {
        if (tid < p.T) s.flags[tid] = head_token_flags(p.tg, tid, p.N);
        if constexpr (LIST)
            for (int i = tid; i < p.T * p.tg.events; i += kFewHeadThreads) s.col[i / p.tg.events][i % p.tg.events] = p.tg.ev_col[i];
    }
}
// A thread's way through the targets of its token, along words that ascend.
template <int NT, bool LIST>
struct FewCursor {
    int e, next;
    __device__ FewCursor(const HeadFewParams& p, const FewTargets<NT, LIST>& s, int tok, bool asked) : e(0), next(kNoColumn) {
        if (LIST && asked) next = s.col[tok][0];
    }
    // Calls at(e) for every target that is word n, one of the WORDS from `first` on.
    template <int WORDS, class At>
    __device__ __forceinline__ void visit(const HeadFewParams& p, const FewTargets<NT, LIST>& s, int tok, int first, int n, At&& at) {
        if constexpr (LIST) {
            while (next < first) { ++e; next = e < p.tg.events ? s.col[tok][e] : kNoColumn; }
            for (int f = e, c = next; c < first + WORDS;) {
                if (c == n) at(f);
                ++f;
                c = f < p.tg.events ? s.col[tok][f] : kNoColumn;
            }
        }
    }
};

// KBW: blocks of 32 columns per warp (K <= 512 KBW).  NT: groups of 8 tokens.  LIST, DUAL as in head_gemm_tcgen05.cuh.
template <int KBW, int NT, bool LIST, bool DUAL>
__global__ void __launch_bounds__(kFewHeadThreads, 1)
head_few_forward_kernel(const HeadFewParams p) {
    constexpr int kTok = 8 * NT;
    __shared__ float s_part[kFewHeadWarps][16][kTok];
    __shared__ FewTargets<NT, LIST> s_tg;
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
    few_targets(p, s_tg, reinterpret_cast<int*>(&s_part[0][0][0]));
    __syncthreads();

    uint4 x[KBW][NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int t = nt * 8 + g;
        const bool there = t < p.T && (s_tg.flags[t] & (kRowDistill | kRowLabel));
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
            const int kb = warp + kFewHeadWarps * i;
            x[i][nt] = make_uint4(0u, 0u, 0u, 0u);
            if (there && kb < kbs) x[i][nt] = __ldg(reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(t) * p.K + kb * 32 + t4 * 8));
        }
    }
    // the word and token of this thread in every block
    const int tok = tid % kTok, slot = tid / kTok;
    const bool asked = slot < 16 && tok < p.T && (s_tg.flags[tok] & (kRowDistill | kRowLabel));
    const int label = !LIST && asked ? static_cast<int>(p.tg.labels[tok]) : -1;
    float m = -INFINITY, s0 = 0.0f, s1 = 0.0f;
    FewCursor<NT, LIST> cursor(p, s_tg, tok, asked);

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
        if (asked && n < p.N) {
            float z = 0.0f;
#pragma unroll
            for (int v = 0; v < kFewHeadWarps; ++v) z += s_part[v][slot][tok];
            const float m_new = fmaxf(m, z);
            s0 = s0 * ex2_approx((m - m_new) * p.c0) + ex2_approx((z - m_new) * p.c0);
            if (DUAL) s1 = s1 * ex2_approx((m - m_new) * p.c1) + ex2_approx((z - m_new) * p.c1);
            m = m_new;
            if (!LIST && n == label) p.z_ev[tok] = z;
            cursor.template visit<16>(p, s_tg, tok, nb * 16, n, [&](int e) { p.z_ev[static_cast<size_t>(tok) * p.tg.events + e] = z; });
        }
        __syncthreads();
    }
    float* red = &s_part[0][0][0];                                  // [3][16][kTok]
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
            if (mq == -INFINITY && sq == 0.0f) continue;           // a slot without words
            a0 += sq * ex2_approx((mq - mm) * p.c0);
            if (DUAL) a1 += red[(32 + q) * kTok + tid] * ex2_approx((mq - mm) * p.c1);
        }
        const size_t at = static_cast<size_t>(tid) * gridDim.x + blockIdx.x;
        p.part[at] = make_float2(mm, a0);
        if (DUAL) p.part1[at] = a1;
    }
}

// Dynamic shared memory: the tokens' rows, 16 bytes apart from a multiple of 128 (an 8 x 8 tile's rows then lie on different
// banks), before that the room of few_targets.  Of every 32 columns the pairs 8 t + 2 j, 8 t + 2 j + 1 lie at 8 j + 2 t: tile j of
// `ldmatrix` is then register j of a lane's 16 bytes, and its transposed form what movmatrix would make of it.
static inline int head_few_x_bytes(int T, int K) { return (T <= 8 ? 8 : 16) * std::max(2 * K + 16, 2 * kFewOwnEvents * 4); }

template <bool TRANS>
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// The shares of 512 columns that a launch is made for, and the words per step that go with them.
static inline int head_few_shares(int K) { return K <= 1024 ? 2 : (K <= 2560 ? 5 : 8); }
__host__ __device__ constexpr int few_backward_words(int kbw, int nt) { return kbw * (8 + 8 * nt) <= 100 ? 16 : 8; }    // dx and words: 4 bytes x this per thread
static inline int head_few_words(int T, int K) { return few_backward_words(head_few_shares(K), T <= 8 ? 1 : 2); }

constexpr float kFewLarge = 0x1p-9f;              // an entry of dz whose second bf16 part matters, in the call's unit

// Words per step: 16 where the registers hold them beside dx (a 16-row MMA is full then, and a step's barriers are spread over twice
// the words), else 8.
template <int KBW, int NT, bool LIST, bool DUAL>
__global__ void __launch_bounds__(kFewHeadThreads, 1)
head_few_backward_kernel(const HeadFewParams p) {
    constexpr int H = few_backward_words(KBW, NT) / 8;
    constexpr int kTok = 8 * NT, kWords = 8 * H;
    constexpr int kParts = kFewHeadThreads / (kWords * kTok) < 4 ? kFewHeadThreads / (kWords * kTok) : 4;   // threads per sum of the warps' parts
    constexpr int kRow = kWords + 2, kPart = kTok * kRow + 2;       // of the parts, in floats: what is read or written at once lies on all banks
    constexpr float kLog2e = 1.4426950408889634f;
    __shared__ float s_part[kFewHeadWarps * kPart];
    __shared__ FewTargets<NT, LIST> s_tg;
    __shared__ float4 s_k[kTok];                                    // -lse log2(e) and gradient per loss (registers are for dx)
    __shared__ int s_label[kTok];
    __shared__ int2 s_cursor[kFewHeadWarps];                        // a warp's token's next target and its word
    // dz in bf16, and what that leaves off as well, in bf16 again: with few tokens a value of dW is a few products, and a gradient's
    // own rounding to bf16 should be the only one that shows (1.7e-3 instead of 1.7e-3 to 3.7e-3 in the 2-norm; 8 tokens leave
    // half of an MMA's indices free for it, 4 % of the time of a step).  For 16 tokens of more than 1024 columns dW gets the second part only in
    // steps where an entry of dz is at least kFewLarge in the call's unit, that is where targets are: smaller ones make a gradient by the hundreds, and
    // what they leave off averages out.  In every step it took 30 % longer (16 x 2560 x 32000 143 us; now 121, 111 without)
    constexpr bool kSome = NT == 2 && KBW > 2;
    constexpr int kSplit = 2, kAlways = kSome ? 1 : 2;
    __shared__ __align__(16) uint16_t s_dz[kSplit][kTok][kWords];   // B operand of dx: pairs of words of a token
    __shared__ __align__(16) uint16_t s_dzt[kSplit][kWords][kTok];  // A operand of dW: pairs of tokens of a word
    extern __shared__ __align__(16) uint8_t s_x[];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    const int blocks = (p.N + kWords - 1) / kWords, kbs = p.K >> 5, pitch = 2 * p.K + 16;

    uint4 w[KBW][H];
    auto load_block = [&](int i, int nb) {
        const int kb = warp + kFewHeadWarps * i;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int n = nb * kWords + h * 8 + g;
            w[i][h] = make_uint4(0u, 0u, 0u, 0u);
            if (kb < kbs && nb < blocks && n < p.N) w[i][h] = load_stream(p.w + static_cast<size_t>(n) * p.K + kb * 32 + t4 * 8);
        }
    };
#pragma unroll
    for (int i = 0; i < KBW; ++i) load_block(i, blockIdx.x);
    few_targets(p, s_tg, reinterpret_cast<int*>(s_x));
    __syncthreads();
    const float unit = head_scale_unit(warp_max(lane < p.T ? head_scale_share(p.scale, LIST, s_tg.flags[lane], lane) : 0.0f));
    if (blockIdx.x == 0 && tid == 0) p.scale.out[0] = unit;
    const int vecs = p.K >> 3;
    for (int i = tid; i < kTok * vecs; i += kFewHeadThreads) {
        const int t = i / vecs, c = i - t * vecs;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (t < p.T && (s_tg.flags[t] & (kRowDistill | kRowLabel))) v = __ldg(reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(t) * p.K) + c);
        uint32_t* to = reinterpret_cast<uint32_t*>(s_x + t * pitch + (c >> 2) * 64 + (c & 3) * 4);
        to[0] = v.x; to[4] = v.y; to[8] = v.z; to[12] = v.w;
    }
    if (tid < kTok) {
        const int flags = tid < p.T ? s_tg.flags[tid] : 0;
        float4 k = make_float4(-INFINITY, 0.0f, -INFINITY, 0.0f);
        if (!LIST && blockIdx.x == 0) report_bad(flags);
        if (flags & (LIST ? kRowDistill : kRowLabel)) {
            k.x = -p.lse0[tid] * kLog2e;
            k.y = p.scale.g0[tid] * p.inv_tau / unit;
        }
        if (DUAL && (flags & kRowLabel)) {
            k.z = -p.lse1[tid] * kLog2e;
            k.w = p.scale.g1[tid] / unit;
        }
        s_k[tid] = k;
        s_label[tid] = !LIST && (flags & kRowLabel) ? static_cast<int>(p.tg.labels[tid]) : -1;
    }
    if (LIST && lane == 0 && tid < kTok * kWords * kParts) {
        const int tok = tid / (kWords * kParts);
        s_cursor[warp] = make_int2(0, tok < p.T && s_tg.flags[tok] != 0 ? s_tg.col[LIST ? tok : 0][0] : kNoColumn);
    }
    __syncthreads();

    // ldmatrix: lane's row lane % 8 (a token) of tile lane / 8
    const uint32_t x_lane = smem_u32(s_x) + static_cast<uint32_t>((lane & 7) * pitch + (lane >> 3) * 16);
    float acc[KBW][2][NT][4] = {};
    for (int nb = blockIdx.x; nb < blocks; nb += gridDim.x) {
        {
            // the words after the next ones: on their way from memory to the L2 while these are worked on
            const long long n = (static_cast<long long>(nb) + 2ll * gridDim.x) * kWords + tid;
            if (tid < kWords && n < p.N) prefetch_l2_bulk(p.w + static_cast<size_t>(n) * p.K, static_cast<uint32_t>(2 * p.K));
        }
        float d[H][2][4] = {};                                      // D rows: tokens g, g + 8; columns: words 2 t, 2 t + 1; two chains
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
            const int kb = warp + kFewHeadWarps * i;
            if (kb < kbs) {
                uint32_t a[4], b[4] = {};
                ldmatrix_x4<false>(a, x_lane + kb * 64);
                if (NT == 2) ldmatrix_x4<false>(b, x_lane + 8 * pitch + kb * 64);
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    mma_bf16_k16(d[h][0], a[0], b[0], a[1], b[1], w[i][h].x, w[i][h].y);
                    mma_bf16_k16(d[h][1], a[2], b[2], a[3], b[3], w[i][h].z, w[i][h].w);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
            float* to = &s_part[warp * kPart + g * kRow + h * 8 + 2 * t4];
            *reinterpret_cast<float2*>(to) = make_float2(d[h][0][0] + d[h][1][0], d[h][0][1] + d[h][1][1]);
            if (NT == 2) *reinterpret_cast<float2*>(to + 8 * kRow) = make_float2(d[h][0][2] + d[h][1][2], d[h][0][3] + d[h][1][3]);
        }
        __syncthreads();
        bool large = false;
        if (tid < kTok * kWords * kParts) {                         // whole warps, a token each
            const int tok = tid / (kWords * kParts), slot = tid / kParts % kWords, part = tid % kParts;
            const int n = nb * kWords + slot;
            float z = 0.0f;
#pragma unroll
            for (int q = 0; q < kFewHeadWarps / kParts; ++q) z += s_part[(kFewHeadWarps / kParts * part + q) * kPart + tok * kRow + slot];
#pragma unroll
            for (int o = 1; o < kParts; o <<= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, o);
            const float4 k = s_k[tok];
            float v = ex2_approx(fmaf(z, p.c0, k.x)) * k.y;
            if (DUAL) v = fmaf(ex2_approx(fmaf(z, p.c1, k.z)), k.w, v);
            if constexpr (LIST) {
                int2 cur = s_cursor[warp];
                if (cur.y < (nb + 1) * kWords) {                    // the same for the warp
                    while (cur.y < nb * kWords) { ++cur.x; cur.y = cur.x < p.tg.events ? s_tg.col[tok][cur.x] : kNoColumn; }
                    for (int f = cur.x, c = cur.y; c < (nb + 1) * kWords;) {
                        if (c == n) {
                            const float q = p.job.index != nullptr ? s_tg.w[tok][f] : p.tg.ev_w[static_cast<size_t>(tok) * p.tg.events + f];
                            v -= q < 0.0f ? k.w : q * k.y;
                        }
                        ++f;
                        c = f < p.tg.events ? s_tg.col[tok][f] : kNoColumn;
                    }
                    __syncwarp();
                    if (lane == 0) s_cursor[warp] = cur;
                }
            } else if (n == s_label[tok]) {
                v -= k.y;
            }
            if (n >= p.N || (k.y == 0.0f && k.w == 0.0f)) v = 0.0f;   // behind the vocabulary; nothing asked (z may be anything)
            large = fabsf(v) >= kFewLarge;
#pragma unroll
            for (int q = 0; q < kSplit; ++q) {
                unsigned short o;
                asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(o) : "f"(v));
                if (part == 0) {
                    s_dz[q][tok][slot] = o;
                    s_dzt[q][slot][tok] = o;
                }
                v -= __uint_as_float(static_cast<uint32_t>(o) << 16);
            }
        }
        if constexpr (kSome) large = __syncthreads_or(large);
        else __syncthreads();
        if constexpr (kSome) {
            static_assert(!kSome || H == 1, "one row of words per lane");
            if (large && p.dw != nullptr) {
                // dW of this step, with both parts
                uint32_t t_dz[2][NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    t_dz[0][nt] = *reinterpret_cast<const uint32_t*>(&s_dzt[0][g][nt * 8 + 2 * t4]);
                    t_dz[1][nt] = *reinterpret_cast<const uint32_t*>(&s_dzt[1][g][nt * 8 + 2 * t4]);
                }
                const int n = nb * kWords + g;
#pragma unroll
                for (int i = 0; i < KBW; ++i) {
                    const int kb = warp + kFewHeadWarps * i;
                    if (kb < kbs) {
                        uint32_t lo[4], hi[4], o[4];
                        ldmatrix_x4<true>(lo, x_lane + kb * 64);
                        ldmatrix_x4<true>(hi, x_lane + 8 * pitch + kb * 64);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float e[4] = {};
#pragma unroll
                            for (int k = 0; k < 2; ++k) mma_bf16_k16(e, t_dz[k][0], 0u, t_dz[k][NT - 1], 0u, lo[j], hi[j]);
                            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[j]) : "f"(e[1] * unit), "f"(e[0] * unit));
                        }
                        if (n < p.N) *reinterpret_cast<uint4*>(p.dw + static_cast<size_t>(n) * p.K + kb * 32 + t4 * 8) = make_uint4(o[0], o[1], o[2], o[3]);
                        __syncwarp();
                    }
                }
            }
        }
        const bool write_dw = p.dw != nullptr && !(kSome && large);
        uint32_t dz[kSplit][NT][H], dzt[kAlways][NT][2] = {};
#pragma unroll
        for (int q = 0; q < kSplit; ++q)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    dz[q][nt][h] = *reinterpret_cast<const uint32_t*>(&s_dz[q][nt * 8 + g][h * 8 + 2 * t4]);
                    if (q < kAlways) dzt[q < kAlways ? q : 0][nt][h] = *reinterpret_cast<const uint32_t*>(&s_dzt[q][h * 8 + g][nt * 8 + 2 * t4]);
                }
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
            const int kb = warp + kFewHeadWarps * i;
            if (kb < kbs) {                                         // the same for the whole warp
                if (p.acc != nullptr) {
                    const uint32_t lo[4] = {w[i][0].x, w[i][0].y, w[i][0].z, w[i][0].w};
                    const uint32_t hi[4] = {w[i][H - 1].x, w[i][H - 1].y, w[i][H - 1].z, w[i][H - 1].w};
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t a0 = transpose_8x8(lo[2 * q]), a1 = transpose_8x8(lo[2 * q + 1]);
                        if constexpr (H == 2) {
                            const uint32_t a2 = transpose_8x8(hi[2 * q]), a3 = transpose_8x8(hi[2 * q + 1]);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int k = 0; k < kSplit; ++k) mma_bf16_k16(acc[i][q][nt], a0, a1, a2, a3, dz[k][nt][0], dz[k][nt][H - 1]);
                        } else {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_bf16_k16(acc[i][q][nt], a0, a1, a0, a1, dz[0][nt][0], dz[1][nt][0]);
                            }
                        }
                    }
                }
                load_block(i, nb + static_cast<int>(gridDim.x));
                if (write_dw) {
                    uint32_t lo[4], hi[4];
                    ldmatrix_x4<true>(lo, x_lane + kb * 64);
                    if (NT == 2) ldmatrix_x4<true>(hi, x_lane + 8 * pitch + kb * 64);
                    uint32_t o[H][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float e[4] = {};
                        if constexpr (NT == 1) {
                            mma_bf16_k16(e, dzt[0][0][0], dzt[0][0][1], dzt[kAlways - 1][0][0], dzt[kAlways - 1][0][1], lo[j], lo[j]);
                        } else {
#pragma unroll
                            for (int k = 0; k < kAlways; ++k) mma_bf16_k16(e, dzt[k][0][0], dzt[k][0][1], dzt[k][NT - 1][0], dzt[k][NT - 1][1], lo[j], hi[j]);
                        }
#pragma unroll
                        for (int h = 0; h < H; ++h)
                            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[h][j]) : "f"(e[2 * h + 1] * unit), "f"(e[2 * h] * unit));
                    }
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        const int n = nb * kWords + h * 8 + g;
                        if (n < p.N) *reinterpret_cast<uint4*>(p.dw + static_cast<size_t>(n) * p.K + kb * 32 + t4 * 8) = make_uint4(o[h][0], o[h][1], o[h][2], o[h][3]);
                    }
                    __syncwarp();
                }
            }
        }
    }
    if (p.acc == nullptr) return;
    // The sums of 4 NT tokens at a time through shared memory (where x was), so that rows leave whole: as the lanes have them, 8 bytes
    // of a sector at a time, they took 17 us for 16 tokens x 2560.
    float* rows = reinterpret_cast<float*>(s_x);
    float* to = p.acc + static_cast<size_t>(blockIdx.x) * p.T * p.K;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KBW; ++i) {
            const int kb = warp + kFewHeadWarps * i;
            if (kb < kbs) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // D row g or g + 8 = j 2 q or 2 q + 1, its column g / 2 * 8 + 2 j + g % 2 of the block; D column = token
                            const int c = kb * 32 + (g >> 1) * 8 + 2 * (2 * q + (e >> 1)) + (g & 1), t = nt * 8 + 2 * t4 + (e & 1) - half * 4 * NT;
                            if (t >= 0 && t < 4 * NT) rows[t * p.K + c] = acc[i][q][nt][e];
                        }
            }
        }
        __syncthreads();
        const int count = min(4 * NT, p.T - half * 4 * NT) * (p.K >> 2);
        float4* out = reinterpret_cast<float4*>(to + static_cast<size_t>(half) * 4 * NT * p.K);
        for (int i = tid; i < count; i += kFewHeadThreads) out[i] = reinterpret_cast<const float4*>(rows)[i];
    }
}

}  // namespace sbn
