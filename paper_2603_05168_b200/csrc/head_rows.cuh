// Losses at the output head, what is done per token (the products are in head_gemm_tcgen05.cuh):
//
//   head_targets_kernel   distillation: the teacher's entries of a row become probabilities q = softmax(l / tau), sorted by
//                         index together with the label, so that a GEMM tile finds those that fall into its columns
//   head_rows_kernel      which rows count at all.  Rows that nothing is asked of (label < 0, no teacher entries: padding,
//                         prompts) are left out of every product: the rows that count move together, in their order, when
//                         any is left out, so such rows cost no work and whatever they hold -- NaN, infinities -- reaches
//                         nothing.  The count stays on the device; the GEMM kernels read it
//   head_losses_kernel    log-sum-exp and losses from the partial maxima and sums of the logits kernel
//   head_dx_kernel        sums of dx in fp32 -> bf16, back at the tokens' own rows, zeros in rows left out
//
// All memory-bound or latency-bound and small beside the products (4096 tokens: 2 to 10 us each).  No atomics: every result
// is the same from run to run.
#pragma once

#include "sbn_common.cuh"

namespace sbn {

constexpr int kHeadMaxTop = 256;                  // teacher entries per token
constexpr int kNoColumn = 0x7FFFFFFF;             // an event that is not there: behind every column

// What is asked of a row, and what is wrong with it.
constexpr int kRowDistill = 1, kRowLabel = 2, kRowBadTeacher = 4, kRowBadLabel = 8;

// What a row's gradient or loss refers to.  Cross entropy: the label.  Distillation: `events` entries per row, sorted by
// column; weight >= 0 is a teacher probability, -1 marks the label's entry.
struct HeadTargets {
    const long long* labels;                      // [T] or null
    const unsigned char* flags;                   // [T], distillation only
    const int* ev_col;                            // [T][events]
    const float* ev_w;
    const int* ev_top;                            // [T]: the entry with the largest probability
    int events;
};

// What is asked of token t.
__device__ __forceinline__ int head_token_flags(const HeadTargets& tg, int t, int N) {
    if (tg.flags != nullptr) return tg.flags[t];
    const long long y = tg.labels[t];
    return y < 0 ? 0 : (y < N ? kRowLabel : kRowBadLabel);
}
// Only where nothing is recorded: a wait that ran out is the graver fault (whole results, not a row) and overwrites this one.
__device__ __forceinline__ void report_bad(int flags) {
    if (flags & (kRowBadTeacher | kRowBadLabel)) atomicCAS(&g_device_status, 0, static_cast<int>(SBN_ERR_INDEX));
}
// A token left out: the outputs of a forward call (any pointer may be null; distillation 0, label 1), and what is wrong with it.
__device__ __forceinline__ void write_left_out(float* loss0, float* loss1, float* lse0, float* lse1, int t, int flags) {
    const float nan = __uint_as_float(0x7FC00000u);
    if (loss0 != nullptr) loss0[t] = (flags & kRowBadTeacher) ? nan : 0.0f;
    if (loss1 != nullptr) loss1[t] = (flags & kRowBadLabel) ? nan : 0.0f;
    if (lse0 != nullptr) lse0[t] = 0.0f;
    if (lse1 != nullptr) lse1[t] = 0.0f;
    report_bad(flags);
}

// The unit of dz: the largest |gradient of a loss| of the call (times 1 / tau for the distillation); 1 if that is none.
// Kept as {unit, 1 / unit}.
struct HeadScale {
    const float *g0, *g1;                         // gradients per token (g1 may be null)
    float inv_tau;
    float* out;                                   // [2]
};
// A token's part in the maximum; what is not asked of it does not count.
__device__ __forceinline__ float head_scale_share(const HeadScale& s, bool distill, int flags, int t) {
    float m = 0.0f;
    if (flags & (distill ? kRowDistill : kRowLabel)) m = fabsf(s.g0[t]) * s.inv_tau;
    if (s.g1 != nullptr && (flags & kRowLabel)) m = fmaxf(m, fabsf(s.g1[t]));
    return m;
}
__device__ __forceinline__ float head_scale_unit(float largest) { return largest > 0x1p-100f && largest < 0x1p100f ? largest : 1.0f; }

struct HeadTargetsJob {
    const long long* index;                       // [T][top]
    const void* logits;                           // [T][top] fp32 or bf16
    int logits_bf16, top, T, N;
    float inv_tau;
    const long long* labels;                      // or null
    unsigned char* flags;
    int* ev_col;
    float* ev_w;
    int* ev_top;
};

// A token's targets, by a warp: flags; put(place, column, weight) gets the entries in order; *top_place: of the heaviest one.  col, val: shared memory for top + 1
// and top entries.  The place of an entry is the number of entries before it (column, then position): top is at most 256, so
// counting costs less than a sorting network's exchanges would.
template <class Put>
__device__ __forceinline__ int warp_targets(const HeadTargetsJob& j, long long t, int lane, int* col, float* val, int* top_place, Put&& put) {
    const int events = j.top + (j.labels != nullptr ? 1 : 0);
    const long long* index = j.index + t * j.top;
    float top_val = -INFINITY;
    int bad = 0, any = 0;
    for (int i = lane; i < j.top; i += 32) {
        const long long c = index[i];
        const float l = j.logits_bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(j.logits)[t * j.top + i]) << 16)
                                      : static_cast<const float*>(j.logits)[t * j.top + i];
        const bool there = c >= 0 && c < j.N;
        bad |= c >= j.N;
        any |= there && !(l == -INFINITY);                   // a NaN counts, and shows in the loss
        col[i] = there ? static_cast<int>(c) : kNoColumn;
        val[i] = there ? l : -INFINITY;
        if (there) top_val = fmaxf(top_val, l);
    }
    top_val = warp_max(top_val);
    bad = __any_sync(0xFFFFFFFFu, bad);
    any = __any_sync(0xFFFFFFFFu, any) && !bad;
    float sum = 0.0f;
    for (int i = lane; i < j.top; i += 32) {
        // the difference first: the type's lowest value, divided by a small temperature, would become -inf
        const float e = val[i] == -INFINITY ? 0.0f : expf((val[i] - top_val) * j.inv_tau);
        val[i] = e;
        sum += e;
        if (!any) col[i] = kNoColumn;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    int flags = (any ? kRowDistill : 0) | (bad ? kRowBadTeacher : 0);
    if (j.labels != nullptr) {
        const long long y = j.labels[t];
        flags |= y < 0 ? 0 : (y < j.N ? kRowLabel : kRowBadLabel);
        if (lane == 0) col[j.top] = (flags & kRowLabel) ? static_cast<int>(y) : kNoColumn;
    }
    __syncwarp();
    int heaviest = kNoColumn;
    for (int i = lane; i < events; i += 32) {
        const int c = col[i];
        int place = 0;
        for (int o = 0; o < events; ++o) place += (col[o] < c || (col[o] == c && o < i)) ? 1 : 0;
        put(place, c, i == j.top ? -1.0f : (c == kNoColumn ? 0.0f : val[i] / sum));
        if (i < j.top && c != kNoColumn && val[i] == 1.0f) heaviest = min(heaviest, place);    // exp of nothing: the largest logit
    }
    heaviest = __reduce_min_sync(0xFFFFFFFFu, heaviest);
    *top_place = heaviest < events ? heaviest : 0;           // (none if a logit is no number)
    return flags;
}

constexpr int kTargetWarps = 4;

// A warp per token.
__global__ void __launch_bounds__(32 * kTargetWarps)
head_targets_kernel(const HeadTargetsJob j) {
    __shared__ int s_col[kTargetWarps][kHeadMaxTop + 1];
    __shared__ float s_val[kTargetWarps][kHeadMaxTop];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int events = j.top + (j.labels != nullptr ? 1 : 0);
    for (long long t = static_cast<long long>(blockIdx.x) * kTargetWarps + warp; t < j.T; t += static_cast<long long>(gridDim.x) * kTargetWarps) {
        int heaviest;
        const int flags = warp_targets(j, t, lane, s_col[warp], s_val[warp], &heaviest, [&](int place, int c, float w) {
            j.ev_col[t * events + place] = c;
            j.ev_w[t * events + place] = w;
        });
        if (lane == 0) {
            j.flags[t] = static_cast<unsigned char>(flags);
            j.ev_top[t] = heaviest;
            report_bad(flags);
        }
        __syncwarp();
    }
}

struct HeadRowsJob {
    HeadTargets tg;
    const uint16_t* x;                            // [T][K]
    int T, K, N;
    int* count;                                   // out: number of rows that count
    int* row_src;                                 // out [T]: token of row r
    int* row_of;                                  // out [T] or null: row of token t, -1 if left out
    uint16_t* xc;                                 // out [T up to a multiple of 64][K], written only if rows are left out
    float *loss0, *loss1, *lse0, *lse1;           // forward: outputs of rows left out (all null: backward)
    HeadScale scale;                              // backward (out null: forward)
};

constexpr int kRowsThreads = 256;

// Sum of v over the block; every thread gets it.
__device__ __forceinline__ int block_sum(int v, int* scratch) {
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < kRowsThreads / 32; ++w) s += scratch[w];
    return s;
}

// CTA b has tokens [b per, (b + 1) per).  Every CTA counts all tokens itself (8 or 1 bytes each, from the L2) instead of
// waiting for the others' counts: one launch, nothing to order.
__global__ void __launch_bounds__(kRowsThreads)
head_rows_kernel(const HeadRowsJob j, const int per) {
    __shared__ int s_scratch[kRowsThreads / 32];
    __shared__ float s_largest[kRowsThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int first = blockIdx.x * per, last = min(j.T, first + per);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int before = 0, total = 0;
    float largest = 0.0f;
    for (int t = tid; t < j.T; t += kRowsThreads) {
        const int c = (head_token_flags(j.tg, t, j.N) & (kRowDistill | kRowLabel)) ? 1 : 0;
        total += c;
        before += t < first ? c : 0;
        if (blockIdx.x == 0 && j.scale.out != nullptr) largest = fmaxf(largest, head_scale_share(j.scale, j.tg.flags != nullptr, head_token_flags(j.tg, t, j.N), t));
    }
    if (blockIdx.x == 0 && j.scale.out != nullptr) {
        largest = warp_max(largest);
        if (lane == 0) s_largest[warp] = largest;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kRowsThreads / 32; ++w) largest = fmaxf(largest, s_largest[w]);
            j.scale.out[0] = head_scale_unit(largest);
            j.scale.out[1] = 1.0f / head_scale_unit(largest);
        }
    }
    total = block_sum(total, s_scratch);
    before = block_sum(before, s_scratch);
    if (blockIdx.x == 0 && tid == 0) *j.count = total;
    for (int t0 = first; t0 < last; t0 += kRowsThreads) {
        const int t = t0 + tid;
        const int flags = t < last ? head_token_flags(j.tg, t, j.N) : 0;
        const bool counts = (flags & (kRowDistill | kRowLabel)) != 0;
        const unsigned ballot = __ballot_sync(0xFFFFFFFFu, counts);
        __syncthreads();
        if (lane == 0) s_scratch[warp] = __popc(ballot);
        __syncthreads();
        int r = before, all = 0;
#pragma unroll
        for (int w = 0; w < kRowsThreads / 32; ++w) {
            r += w < warp ? s_scratch[w] : 0;
            all += s_scratch[w];
        }
        r += __popc(ballot & ((1u << lane) - 1u));
        if (counts) j.row_src[r] = t;
        if (t < last) {
            if (j.row_of != nullptr) j.row_of[t] = counts ? r : -1;
            if (!counts) {
                write_left_out(j.loss0, j.loss1, j.lse0, j.lse1, t, flags);
            }
        }
        if (total < j.T) {
            // the rows that count, 16 bytes at a time, one row after another
            __syncthreads();
            const int vecs = j.K >> 3;
            uint4* to = reinterpret_cast<uint4*>(j.xc + static_cast<size_t>(before) * j.K);
#pragma unroll 4
            for (int v = tid; v < all * vecs; v += kRowsThreads) {           // at most 256 rows of 2^20 values: below 2^25
                const int i = v / vecs;
                to[v] = __ldg(reinterpret_cast<const uint4*>(j.x + static_cast<size_t>(j.row_src[before + i]) * j.K) + (v - i * vecs));
            }
        }
        before += all;
    }
    if (total < j.T && blockIdx.x == gridDim.x - 1) {
        // dW contracts over whole stages of 64 rows: zeros behind the last row that counts
        const int rows = ((max(total, 1) + 63) & ~63) - total, vecs = j.K >> 3;
        uint4* to = reinterpret_cast<uint4*>(j.xc + static_cast<size_t>(total) * j.K);
        for (long long v = tid; v < static_cast<long long>(rows) * vecs; v += kRowsThreads) to[v] = make_uint4(0u, 0u, 0u, 0u);
    }
}

struct HeadLossJob {
    HeadTargets tg;
    const int* count;                             // null (few tokens): every token has its row
    const int* row_src;
    int T, N;
    const float2* part;                           // [rows][parts]: maximum m of the raw logits, sum of exp((z - m) / tau)
    const float* part1;                           // [rows][parts] or null: sum of exp(z - m)
    const float* z_ev;                            // [rows][events]: logits at the targets
    const uint16_t *x, *w;
    int K;
    int parts;
    double inv_tau;
    double z_scale;                               // of the logits in part and z_ev (head_logit_scale)
    float *loss0, *loss1, *lse0, *lse1;           // at the tokens' own rows: distillation, label.  Cross entropy: loss1 and lse0
};

constexpr int kLossThreads = 128;

// A thread's share of x[t] . w[word].
__device__ __forceinline__ float head_logit_share(const HeadLossJob& j, int t, long long word, int tid) {
    const uint4* a = reinterpret_cast<const uint4*>(j.x + static_cast<size_t>(t) * j.K);
    const uint4* b = reinterpret_cast<const uint4*>(j.w + static_cast<size_t>(word) * j.K);
    float lo = 0.0f, hi = 0.0f;
#pragma unroll 4
    for (int i = tid; i < j.K >> 3; i += kLossThreads) {
        const uint4 u = __ldg(a + i), v = __ldg(b + i);
        lo = fmaf(bf16lo_to_f32(u.x), bf16lo_to_f32(v.x), lo); hi = fmaf(bf16hi_to_f32(u.x), bf16hi_to_f32(v.x), hi);
        lo = fmaf(bf16lo_to_f32(u.y), bf16lo_to_f32(v.y), lo); hi = fmaf(bf16hi_to_f32(u.y), bf16hi_to_f32(v.y), hi);
        lo = fmaf(bf16lo_to_f32(u.z), bf16lo_to_f32(v.z), lo); hi = fmaf(bf16hi_to_f32(u.z), bf16hi_to_f32(v.z), hi);
        lo = fmaf(bf16lo_to_f32(u.w), bf16lo_to_f32(v.w), lo); hi = fmaf(bf16hi_to_f32(u.w), bf16hi_to_f32(v.w), hi);
    }
    return lo + hi;
}

// lse - z of one word: log(sum / term), with the term itself taken from the word's exact logit.  sum: of exp of all logits in
// units of exp of the largest, with the word's as the products had it (`was`, relative to the largest); ahead: the largest less the exact logit.
// The rest of the sum is at least 0 (a sum that holds the largest term is never rounded below it), and so is the result: with lse
// and the logit from different sums, a sure token's loss was what their errors differed by: up to 1.1e-4 at 4096 columns, mostly below 0.
// (expf: 1 exactly for the largest term, and where another one is the largest its error is beside a rest of at least 1.)
__device__ __forceinline__ double surprise(double sum, float was, double ahead) {
    double rest = sum - static_cast<double>(expf(was));
    rest = rest < 0.0 ? 0.0 : rest;                           // (a NaN stays)
    if (ahead > 700.0) return ahead + log(rest);
    const double y = rest * exp(ahead);
    return y < 0x1p-10 ? y * (1.0 + y * (-1.0 / 2 + y * (1.0 / 3 - y * (1.0 / 4)))) : log(1.0 + y);      // log1p: off by less than 2^-42 of itself
}

// A CTA per row, everything it reads under way at once: a call with few rows waits for latencies only.  Sums in double: a loss
// is the small difference of two numbers near each other, and this is a few hundred operations per token.
__global__ void __launch_bounds__(kLossThreads)
head_losses_kernel(const HeadLossJob j) {
    constexpr int kWarps = kLossThreads / 32;
    __shared__ float s_f[2][kWarps];
    __shared__ double s_d[6][kWarps];
    __shared__ float s_was[2];                                // logits of the products: the teacher's heaviest entry's, the label's
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows = j.count != nullptr ? *j.count : j.T;
    const float tau_f = static_cast<float>(j.inv_tau * j.z_scale), one_f = static_cast<float>(j.z_scale);
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const int t = j.count != nullptr ? j.row_src[r] : r;
        const int flags = head_token_flags(j.tg, t, j.N);
        if (!(flags & (kRowDistill | kRowLabel))) {           // few tokens only: rows left out are no rows otherwise
            if (tid == 0) write_left_out(j.loss0, j.loss1, j.lse0, j.lse1, t, flags);
            continue;
        }
        const size_t p0 = static_cast<size_t>(r) * j.parts;
        // maxima and sums, as many parts per thread as there are; parts without columns of the vocabulary hold (-inf, 0)
        float m = -INFINITY, s0 = 0.0f, s1 = 0.0f;
        const float2 none = make_float2(-INFINITY, 0.0f);
        for (int i = tid; i < j.parts; i += 4 * kLossThreads) {
            float2 v[4];
            float w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool in = i + q * kLossThreads < j.parts;
                v[q] = in ? j.part[p0 + i + q * kLossThreads] : none;
                w[q] = in && j.part1 != nullptr ? j.part1[p0 + i + q * kLossThreads] : 0.0f;
            }
            const float top = fmaxf(fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x)), m);
            if (top == -INFINITY) {                           // nothing yet; sums that are no numbers stay so
                s0 += (v[0].y + v[1].y) + (v[2].y + v[3].y);
                s1 += (w[0] + w[1]) + (w[2] + w[3]);
                continue;
            }
            s0 *= expf((m - top) * tau_f);
            s1 *= expf((m - top) * one_f);
            m = top;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                s0 += v[q].y * expf((v[q].x - m) * tau_f);
                s1 += w[q] * expf((v[q].x - m) * one_f);
            }
        }
        // The logits of the label and of the teacher's heaviest entry once more, in fp32 on the ordinary units: the tensor cores cut
        // every partial sum off, always towards zero, which is no matter in lse but shows in a loss that is mostly a large logit.
        float dot = 0.0f, dot_top = 0.0f;
        int heaviest = -1;
        if (flags & kRowLabel) dot = head_logit_share(j, t, j.tg.labels[t], tid);
        if (flags & kRowDistill) {
            heaviest = j.tg.ev_top[t];
            dot_top = head_logit_share(j, t, j.tg.ev_col[static_cast<size_t>(t) * j.tg.events + heaviest], tid);
        }
        // the teacher's entries: sum of q, and of q (log q - z / tau) without the heaviest's z.  The label's logit as the products had it
        // goes to whoever needs it in the end
        double q_sum = 0.0, kd = 0.0;
        float q_top = 0.0f;
        if (j.tg.flags != nullptr) {
            for (int i = tid; i < j.tg.events; i += kLossThreads) {
                if (j.tg.ev_col[static_cast<size_t>(t) * j.tg.events + i] == kNoColumn) continue;
                const float q = j.tg.ev_w[static_cast<size_t>(t) * j.tg.events + i];
                const float z_tc = j.z_ev[static_cast<size_t>(r) * j.tg.events + i];
                if (q < 0.0f) s_was[1] = z_tc;                // the label's entry
                if (i == heaviest) s_was[0] = z_tc;
                if (!(q <= 0.0f)) {
                    const double z = i == heaviest ? 0.0 : static_cast<double>(z_tc) * j.z_scale;
                    q_sum += static_cast<double>(q);
                    kd += static_cast<double>(q) * (static_cast<double>(logf(q)) - z * j.inv_tau);
                    if (i == heaviest) q_top = q;
                }
            }
        } else if (tid == 0) {
            s_was[1] = j.z_ev[r];
        }
        const float m_warp = warp_max(m);
        if (lane == 0) s_f[0][warp] = m_warp;
        __syncthreads();
        float top = s_f[0][0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_f[0][w]);
        // no part: s0 and s1 are 0 or no numbers
        const float down0 = m == -INFINITY ? 1.0f : expf((m - top) * tau_f), down1 = m == -INFINITY ? 1.0f : expf((m - top) * one_f);
        double sums[6] = {static_cast<double>(s0) * static_cast<double>(down0), static_cast<double>(s1) * static_cast<double>(down1), q_sum, kd,
                          static_cast<double>(dot_top), static_cast<double>(q_top)};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
#pragma unroll
            for (int k = 0; k < 6; ++k) sums[k] += __shfl_xor_sync(0xFFFFFFFFu, sums[k], o);
        }
        if (lane == 0) {
            s_f[1][warp] = dot;
#pragma unroll
            for (int k = 0; k < 6; ++k) s_d[k][warp] = sums[k];
        }
        __syncthreads();
        // a warp per output: logarithms in double take their time one after another
        if (lane == 0) {
            dot = s_f[1][0];
#pragma unroll
            for (int k = 0; k < 6; ++k) sums[k] = s_d[k][0];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) {
                dot += s_f[1][w];
#pragma unroll
                for (int k = 0; k < 6; ++k) sums[k] += s_d[k][w];
            }
            const double m_z = static_cast<double>(top) * j.z_scale;
            const bool label_alone = j.tg.flags == nullptr;   // cross entropy: its sum is the first
            const float bad = __uint_as_float(0x7FC00000u);
            if (warp == 0) {
                j.lse0[t] = label_alone || (flags & kRowDistill) ? static_cast<float>(m_z * j.inv_tau + log(sums[0])) : 0.0f;
            } else if (warp == 1) {
                if (j.loss1 != nullptr) {
                    float loss1 = (flags & kRowBadLabel) ? bad : 0.0f;
                    if (flags & kRowLabel) loss1 = static_cast<float>(surprise(label_alone ? sums[0] : sums[1], (s_was[1] - top) * one_f, m_z - dot));
                    j.loss1[t] = loss1;
                }
            } else if (warp == 2) {
                if (!label_alone) {
                    float loss0 = (flags & kRowBadTeacher) ? bad : 0.0f;
                    if (flags & kRowDistill) {
                        // sum of q (log q - log p) with log p_j = (z_j - z_top) / tau - the heaviest's surprise
                        const double z_top = sums[4] * j.inv_tau;
                        loss0 = static_cast<float>(sums[3] + (sums[2] - sums[5]) * z_top +
                                                   sums[2] * surprise(sums[0], (s_was[0] - top) * tau_f, m_z * j.inv_tau - z_top));
                    }
                    j.loss0[t] = loss0;
                }
            } else if (j.lse1 != nullptr) {
                j.lse1[t] = (flags & kRowLabel) ? static_cast<float>(m_z + log(sums[1])) : 0.0f;
            }
        }
        __syncthreads();
    }
}

struct HeadDxJob {
    const int* row_of;                            // null (few tokens): every token has its row
    const float* acc;                             // [slots][rows][K]
    int slots, T, K;
    int rows, rest;                               // rest: rows from a token's to its second part's (dz in two parts), 0: there is none
    const float* scale;                           // the unit of dz
    uint16_t* dx;                                 // [T][K]
};

constexpr int kDxThreads = 256;

// GROUPS threads per 4 values, each with every GROUPS-th slot; their sums are added in the groups' order.  REST: dz in two parts.
template <int GROUPS, bool REST>
__global__ void __launch_bounds__(kDxThreads)
head_dx_kernel(const HeadDxJob j) {
    constexpr int kVecs = kDxThreads / GROUPS;    // of a CTA and step
    __shared__ float4 s_sum[GROUPS > 1 ? kDxThreads : 1];
    pdl_launch_dependents();
    pdl_wait();
    const int vecs = j.K >> 2, group = threadIdx.x / kVecs, mine = threadIdx.x % kVecs;
    const long long all = static_cast<long long>(j.T) * vecs;
    const size_t slot = static_cast<size_t>(j.rows) * j.K, rest = static_cast<size_t>(j.rest) * j.K;
    const float scale = *j.scale;
    for (long long first = static_cast<long long>(blockIdx.x) * kVecs; first < all; first += static_cast<long long>(gridDim.x) * kVecs) {
        const long long i = first + mine;
        const int t = static_cast<int>(i / vecs), c = static_cast<int>(i - static_cast<long long>(t) * vecs);
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i < all) {
            const int r = j.row_of != nullptr ? j.row_of[t] : t;
            if (r >= 0) {
                const float* a = j.acc + static_cast<size_t>(r) * j.K + 4 * c;
#pragma unroll 8
                for (int s = group; s < j.slots; s += GROUPS) {
                    float4 o = *reinterpret_cast<const float4*>(a + s * slot);
                    if constexpr (REST) {
                        const float4 r = *reinterpret_cast<const float4*>(a + s * slot + rest);
                        o.x += r.x; o.y += r.y; o.z += r.z; o.w += r.w;
                    }
                    v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                }
            }
        }
        if constexpr (GROUPS > 1) {
            s_sum[threadIdx.x] = v;
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int g = 1; g < GROUPS; ++g) {
                    const float4 o = s_sum[g * kVecs + mine];
                    v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                }
            }
            __syncthreads();
        }
        if (group == 0 && i < all) {
            uint2 o;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.x) : "f"(v.y * scale), "f"(v.x * scale));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.y) : "f"(v.w * scale), "f"(v.z * scale));
            *reinterpret_cast<uint2*>(j.dx + static_cast<size_t>(t) * j.K + 4 * c) = o;
        }
    }
}

}  // namespace sbn
