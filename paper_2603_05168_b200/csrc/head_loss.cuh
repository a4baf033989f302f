// Host side of the losses at the output head: workspaces, pieces of the vocabulary, launches.  Included by libsbn.cu.
#pragma once

#include "head_few_mma.cuh"

namespace sbn {

// How a call is cut up, from its sizes alone.
struct HeadPlan {
    bool few;                     // head_few_mma.cuh
    bool words;                   // logits by head_words_tcgen05.cuh, gradients as for any number of tokens
    int tokens, groups, word_pairs;   // words: tokens per tile and groups of them, CTA pairs
    int bn, parts;                // forward: columns per tile, partial sums per row
    int piece;                    // backward: columns of dz at a time (a multiple of 512)
    int bn_piece;                 // columns per tile of the pieces' logits
    bool wide_grads;              // gradients in tiles of 512 columns, else 256
    int slots, slot_stages;       // slices of dx's contraction over a piece, and 64-column stages of each
    int rest;                     // dz in two parts: rows from a token's to its second part's (kWordsTwoParts), else 0
    int grad_rows;                // rows that the gradients' products have: the tokens, or both parts
    long long rows64, rows256;    // grad_rows up to a multiple
};

static inline long long head_up(long long v, long long to) { return (v + to - 1) / to * to; }

// Columns per tile of z: as wide as possible (a wide tile reads its rows for more columns), narrower where the tiles would
// not go round.  us per stage and per tile, as measured.
static int head_tile_columns(int T, int cols, int K) {
    static const struct { int bn; double stage, tile; } kShapes[] = {{256, 0.38, 1.0}, {128, 0.33, 1.0}, {64, 0.31, 1.0}};
    if (g_force_token_tile < 0) return g_force_token_tile <= -256 ? 256 : (g_force_token_tile <= -128 ? 128 : 64);
    int best = 256;
    double best_cost = 1e300;
    for (const auto& shape : kShapes) {
        const int bn = shape.bn;
        const double tiles = static_cast<double>(head_up(T, 256) / 256) * ((cols + bn - 1) / bn);
        const double rounds = std::ceil(tiles / kBackwardPairs);
        const double cost = rounds * (shape.stage * (K / 64) + shape.tile);
        if (cost < best_cost * 0.99) { best_cost = cost; best = bn; }
    }
    return best;
}

static HeadPlan head_plan(int T, int N, int K) {
    HeadPlan h{};
    h.grad_rows = T;
    h.few = head_few_takes(T, K);
    if (h.few) {
        h.parts = std::min((N + 15) / 16, kNumSMs);
        h.slots = std::min((N + head_few_words(T, K) - 1) / head_few_words(T, K), kNumSMs);
        return h;
    }
    h.words = T <= kWordsTokens;
    if (T <= kWordsTwoParts) {
        h.rest = static_cast<int>(head_up(T, 64));
        h.grad_rows = 2 * h.rest;
    }
    h.rows64 = head_up(h.grad_rows, 64);
    h.rows256 = head_up(h.grad_rows, 256);
    if (h.words) {
        const int tiles = (N + 255) / 256;
        h.groups = std::max(1, std::min(kBackwardPairs / tiles, (T + 31) / 32));
        h.tokens = static_cast<int>(head_up((T + h.groups - 1) / h.groups, 32));
        h.groups = (T + h.tokens - 1) / h.tokens;
        h.word_pairs = std::min(tiles * h.groups, kBackwardPairs);
    }
    h.bn = head_tile_columns(T, N, K);
    h.parts = h.words ? 8 * h.word_pairs : 2 * ((N + h.bn - 1) / h.bn);
    long long cols = (128ll << 20) / (2 * h.rows256);
    cols = std::max(1024ll, cols / 512 * 512);
    const long long pieces = (N + cols - 1) / cols;
    h.piece = static_cast<int>(head_up((N + pieces - 1) / pieces, 512));
    h.bn_piece = head_tile_columns(T, std::min(N, h.piece), K);
    // gradients in wide tiles where those of dx and dW go round more than once (dW's are short: their number counts by length)
    {
        const double rows = static_cast<double>(h.rows256 / 256), words = (std::min(N, h.piece) + 255) / 256;
        auto cost = [&](int cols_per_tile, double stage, double tile) {
            const double across = (K + cols_per_tile - 1) / cols_per_tile;
            const double dx = std::ceil(rows * across / kBackwardPairs) * (stage * 4 * words + tile);
            const double all = (rows * across * (stage * 4 * words + tile) + words * across * (stage * 4 * rows + tile)) / kBackwardPairs;
            return std::max(dx, all);
        };
        h.wide_grads = rows >= 4 && cost(512, 0.56, 2.0) < cost(256, 0.40, 0.5);
        if (g_force_token_tile < 0) h.wide_grads = g_force_token_tile <= -512;
    }
    const int tile_cols = h.wide_grads ? 512 : 256;
    const long long dx_tiles = h.rows256 / 256 * ((K + tile_cols - 1) / tile_cols);     // 2^34 for the largest sizes that can be asked about
    const int stages = (std::min(h.piece, N) + 63) / 64;
    const int slots = std::max(1, std::min(static_cast<int>((kBackwardPairs + dx_tiles / 2) / dx_tiles), stages));
    h.slot_stages = (stages + slots - 1) / slots;
    h.slots = (stages + h.slot_stages - 1) / h.slot_stages;             // all of them are written by the first piece
    return h;
}

// Workspace of a call, in bytes from its start.
struct HeadWs {
    size_t count, scale, row_src, row_of, flags, ev_col, ev_w, ev_top, xc, z_ev, part, part1, dz, acc, total;
};
static HeadWs head_ws_layout(const HeadPlan& h, bool backward, int T, int K, int top) {
    HeadWs w{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~static_cast<size_t>(255); return here; };
    const size_t t = static_cast<size_t>(T), events = top ? static_cast<size_t>(top) + 1 : 1;
    if (backward) w.scale = take(8);
    if (!h.few && !h.words) {
        w.count = take(4);
        w.row_src = take(4 * t);
        w.row_of = take(4 * t);
    }
    if (top) {
        w.flags = take(t);
        w.ev_col = take(4 * t * events);
        w.ev_w = take(4 * t * events);
        w.ev_top = take(4 * t);
    }
    if (!h.few && !(h.words && !backward)) w.xc = take(2 * static_cast<size_t>(h.rows64) * K);
    if (!backward) {
        w.z_ev = take(4 * t * events);
        w.part = take(8 * t * h.parts);
        if (top) w.part1 = take(4 * t * h.parts);
    } else {
        if (!h.few) w.dz = take(2 * static_cast<size_t>(h.rows256) * h.piece);
        w.acc = take(4 * static_cast<size_t>(h.slots) * h.grad_rows * K);
    }
    w.total = at;
    return w;
}

// What leaves in boxes of 32 rows x 64 bytes, with the 64-byte swizzle in shared memory: dz and dW, bf16 [rows][cols], and the
// sums of dx, fp32 [slots][rows][cols].
static bool encode_out(CUtensorMap* map, const void* base, bool bf16, uint64_t cols, uint64_t rows, uint64_t slots) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const uint64_t es = bf16 ? 2 : 4;
    cuuint64_t dims[3] = {cols, rows, slots};
    cuuint64_t strides[2] = {cols * es, cols * es * rows};
    cuuint32_t box[3] = {static_cast<cuuint32_t>(64 / es), 32u, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, bf16 ? 2 : 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One call of either operator: top == 0 is the cross entropy.
struct HeadCall {
    const void* x;
    int T, K;
    const void* head;
    int N;
    const long long* labels;
    const long long* top_index;
    const void* top_logits;
    int top_bf16, top;
    float tau;
    char* ws;
};

static bool head_encode(const HeadCall& c, const HeadPlan& h, const HeadWs& w, int bn, HeadMaps* maps) {
    const uint64_t k = static_cast<uint64_t>(c.K);
    if (h.words)
        return encode_2d_bf16_sw128(&maps->x, c.x, k, c.T, k, static_cast<uint32_t>(h.tokens / 2)) && encode_2d_bf16_sw128(&maps->w, c.head, k, c.N, k, 128);
    return encode_2d_bf16_sw128(&maps->x, c.x, k, c.T, k, 128) && encode_2d_bf16_sw128(&maps->xc, c.ws + w.xc, k, h.rows64, k, 128) &&
           encode_2d_bf16_sw128(&maps->w, c.head, k, c.N, k, bn / 2);
}

template <int MODE, bool LIST, bool DUAL>
static sbn_status launch_head_logits_as(const HeadMaps& maps, const HeadLogitsParams& p, cudaStream_t stream) {
    using Loop = PairLoop<HeadLogitsWork<MODE, LIST, DUAL>>;
    if (!ensure_dynamic_smem<head_logits_kernel<MODE, LIST, DUAL>>(Loop::kSmemBytes)) return SBN_ERR_CUDA;
    const long long tiles = head_up(p.T, 256) / 256 * ((p.v1 - p.v0 + p.bn - 1) / p.bn);
    const unsigned pairs = static_cast<unsigned>(std::min<long long>(tiles, kBackwardPairs));
    if (launch_kernel(head_logits_kernel<MODE, LIST, DUAL>, dim3(2 * pairs), dim3(Loop::kThreads), Loop::kSmemBytes, stream, maps, p) != cudaSuccess)
        return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}
template <int MODE>
static sbn_status launch_head_logits(const HeadMaps& maps, const HeadLogitsParams& p, bool list, bool dual, cudaStream_t stream) {
    if (!list) return launch_head_logits_as<MODE, false, false>(maps, p, stream);
    return dual ? launch_head_logits_as<MODE, true, true>(maps, p, stream) : launch_head_logits_as<MODE, true, false>(maps, p, stream);
}

template <int MODE, bool LIST, bool DUAL, bool REST>
static sbn_status launch_head_words_as(const HeadMaps& maps, const HeadWordsParams& p, cudaStream_t stream) {
    using Loop = PairLoop<HeadWordsWork<MODE, LIST, DUAL, REST>>;
    if (!ensure_dynamic_smem<head_words_kernel<MODE, LIST, DUAL, REST>>(232448)) return SBN_ERR_CUDA;
    if (launch_kernel(head_words_kernel<MODE, LIST, DUAL, REST>, dim3(2 * p.pairs), dim3(Loop::kThreads), words_smem_bytes(p.tokens), stream, maps, p) != cudaSuccess)
        return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}
template <int MODE, bool LIST, bool DUAL>
static sbn_status launch_head_words_of(const HeadMaps& maps, const HeadWordsParams& p, cudaStream_t stream) {
    if constexpr (MODE == 1)
        if (p.rest != 0) return launch_head_words_as<MODE, LIST, DUAL, true>(maps, p, stream);
    return launch_head_words_as<MODE, LIST, DUAL, false>(maps, p, stream);
}
template <int MODE>
static sbn_status launch_head_words(const HeadMaps& maps, const HeadWordsParams& p, bool list, bool dual, cudaStream_t stream) {
    if (!list) return launch_head_words_of<MODE, false, false>(maps, p, stream);
    return dual ? launch_head_words_of<MODE, true, true>(maps, p, stream) : launch_head_words_of<MODE, true, false>(maps, p, stream);
}

// What is asked of the tokens: the labels themselves, or for a distillation the sorted targets of every token.
// `later`: the job for a kernel that does it itself.
static sbn_status launch_head_targets(const HeadCall& c, const HeadWs& w, HeadTargets* tg, cudaStream_t stream, HeadTargetsJob* later = nullptr) {
    *tg = HeadTargets{c.labels, nullptr, nullptr, nullptr, nullptr, 1};
    if (!c.top) return SBN_OK;
    HeadTargetsJob t{c.top_index, c.top_logits, c.top_bf16, c.top, c.T, c.N, static_cast<float>(1.0 / static_cast<double>(c.tau)), c.labels,
                     reinterpret_cast<unsigned char*>(c.ws + w.flags), reinterpret_cast<int*>(c.ws + w.ev_col),
                     reinterpret_cast<float*>(c.ws + w.ev_w), reinterpret_cast<int*>(c.ws + w.ev_top)};
    *tg = HeadTargets{c.labels, t.flags, t.ev_col, t.ev_w, t.ev_top, c.top + (c.labels ? 1 : 0)};
    if (later && tg->events <= kFewOwnEvents) {
        *later = t;
        return SBN_OK;
    }
    const int blocks = std::min((c.T + kTargetWarps - 1) / kTargetWarps, 16 * device_sm_count());
    if (launch_kernel(head_targets_kernel, dim3(blocks), dim3(32 * kTargetWarps), 0, stream, t) != cudaSuccess) return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}

// The rows that count.
static sbn_status launch_head_rows(const HeadCall& c, const HeadWs& w, HeadRowsJob rows, cudaStream_t stream) {
    rows.x = static_cast<const uint16_t*>(c.x);
    rows.T = c.T;
    rows.K = c.K;
    rows.N = c.N;
    rows.count = reinterpret_cast<int*>(c.ws + w.count);
    rows.row_src = reinterpret_cast<int*>(c.ws + w.row_src);
    rows.xc = reinterpret_cast<uint16_t*>(c.ws + w.xc);
    const int blocks = std::min(c.T, 2 * device_sm_count()), per = (c.T + blocks - 1) / blocks;
    if (launch_kernel(head_rows_kernel, dim3((c.T + per - 1) / per), dim3(kRowsThreads), 0, stream, rows, per) != cudaSuccess) return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}

static sbn_status launch_head_losses(const HeadLossJob& j, cudaStream_t stream) {
    const int blocks = std::min(j.T, 16 * device_sm_count());
    if (launch_kernel(head_losses_kernel, dim3(blocks), dim3(kLossThreads), 0, stream, j) != cudaSuccess) return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}
template <int GROUPS, bool REST>
static sbn_status launch_head_dx_as(const HeadDxJob& j, cudaStream_t stream) {
    constexpr int vecs = kDxThreads / GROUPS;
    const long long steps = (static_cast<long long>(j.T) * (j.K / 4) + vecs - 1) / vecs;
    const int blocks = static_cast<int>(std::min<long long>(steps, 16ll * device_sm_count()));
    if (launch_kernel(head_dx_kernel<GROUPS, REST>, dim3(blocks), dim3(kDxThreads), 0, stream, j) != cudaSuccess) return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}
static sbn_status launch_head_dx(const HeadDxJob& j, cudaStream_t stream) {
    if (j.rest != 0) return j.slots > 4 ? launch_head_dx_as<8, true>(j, stream) : launch_head_dx_as<1, true>(j, stream);
    return j.slots > 4 ? launch_head_dx_as<8, false>(j, stream) : launch_head_dx_as<1, false>(j, stream);
}

// ---- few tokens ------------------------------------------------------------------------------------
template <bool BACKWARD, int KBW, int NT, bool LIST, bool DUAL>
static sbn_status launch_head_few_as(const HeadFewParams& p, int ctas, cudaStream_t stream) {
    cudaError_t err;
    if constexpr (BACKWARD) {
        if (!ensure_dynamic_smem<head_few_backward_kernel<KBW, NT, LIST, DUAL>>(160 * 1024)) return SBN_ERR_CUDA;
        err = launch_kernel(head_few_backward_kernel<KBW, NT, LIST, DUAL>, dim3(ctas), dim3(kFewHeadThreads), head_few_x_bytes(p.T, p.K), stream, p);
    } else {
        err = launch_kernel(head_few_forward_kernel<KBW, NT, LIST, DUAL>, dim3(ctas), dim3(kFewHeadThreads), 0, stream, p);
    }
    if (err != cudaSuccess) return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}
template <bool BACKWARD, int KBW, int NT>
static sbn_status launch_head_few_of(const HeadFewParams& p, int ctas, bool list, bool dual, cudaStream_t stream) {
    if (!list) return launch_head_few_as<BACKWARD, KBW, NT, false, false>(p, ctas, stream);
    return dual ? launch_head_few_as<BACKWARD, KBW, NT, true, true>(p, ctas, stream) : launch_head_few_as<BACKWARD, KBW, NT, true, false>(p, ctas, stream);
}
template <bool BACKWARD>
static sbn_status launch_head_few(const HeadFewParams& p, int ctas, bool list, bool dual, cudaStream_t stream) {
    const int shares = head_few_shares(p.K);
    if (p.T <= 8) {
        if (shares == 2) return launch_head_few_of<BACKWARD, 2, 1>(p, ctas, list, dual, stream);
        if (shares == 5) return launch_head_few_of<BACKWARD, 5, 1>(p, ctas, list, dual, stream);
        return launch_head_few_of<BACKWARD, 8, 1>(p, ctas, list, dual, stream);
    }
    if (shares == 2) return launch_head_few_of<BACKWARD, 2, 2>(p, ctas, list, dual, stream);
    return launch_head_few_of<BACKWARD, 5, 2>(p, ctas, list, dual, stream);
}
static HeadFewParams head_few_params(const HeadCall& c, const HeadTargets& tg) {
    HeadFewParams p{};
    p.tg = tg;
    p.x = static_cast<const uint16_t*>(c.x);
    p.w = static_cast<const uint16_t*>(c.head);
    p.T = c.T; p.N = c.N; p.K = c.K;
    p.c0 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K / kFewHeadWarps) / static_cast<double>(c.tau));     // a warp sums that much
    p.c1 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K / kFewHeadWarps));
    p.inv_tau = static_cast<float>(1.0 / static_cast<double>(c.tau));
    return p;
}

static sbn_status head_few_forward(const HeadCall& c, const HeadPlan& h, float* loss0, float* loss1, float* lse0, float* lse1, cudaStream_t stream) {
    const HeadWs w = head_ws_layout(h, false, c.T, c.K, c.top);
    HeadTargets tg;
    HeadTargetsJob job{};
    sbn_status st = launch_head_targets(c, w, &tg, stream, &job);
    if (st != SBN_OK) return st;
    const bool list = c.top != 0, dual = list && c.labels;
    HeadFewParams p = head_few_params(c, tg);
    p.job = job;
    p.part = reinterpret_cast<float2*>(c.ws + w.part);
    p.part1 = dual ? reinterpret_cast<float*>(c.ws + w.part1) : nullptr;
    p.z_ev = reinterpret_cast<float*>(c.ws + w.z_ev);
    st = launch_head_few<false>(p, h.parts, list, dual, stream);
    if (st != SBN_OK) return st;
    return launch_head_losses(HeadLossJob{tg, nullptr, nullptr, c.T, c.N, p.part, p.part1, p.z_ev, p.x, p.w, c.K, h.parts, 1.0 / static_cast<double>(c.tau),
                                          head_logit_scale(c.K / kFewHeadWarps), loss0, loss1, lse0, lse1},
                              stream);
}

static sbn_status head_few_backward(const HeadCall& c, const HeadPlan& h, const float* lse0, const float* lse1, const float* g0, const float* g1, void* dx,
                                    void* dhead, cudaStream_t stream) {
    const HeadWs w = head_ws_layout(h, true, c.T, c.K, c.top);
    HeadTargets tg;
    HeadTargetsJob job{};
    sbn_status st = launch_head_targets(c, w, &tg, stream, &job);
    if (st != SBN_OK) return st;
    const bool list = c.top != 0, dual = list && c.labels;
    HeadFewParams p = head_few_params(c, tg);
    p.job = job;
    p.lse0 = lse0; p.lse1 = lse1;
    p.scale = HeadScale{g0, g1, p.inv_tau, reinterpret_cast<float*>(c.ws + w.scale)};
    p.dw = static_cast<uint16_t*>(dhead);
    p.acc = dx ? reinterpret_cast<float*>(c.ws + w.acc) : nullptr;
    st = launch_head_few<true>(p, h.slots, list, dual, stream);
    if (st != SBN_OK) return st;
    return dx ? launch_head_dx(HeadDxJob{nullptr, p.acc, h.slots, c.T, c.K, c.T, 0, p.scale.out, static_cast<uint16_t*>(dx)}, stream) : SBN_OK;
}

// ---- any number of tokens --------------------------------------------------------------------------
static sbn_status head_forward(const HeadCall& c, float* loss0, float* loss1, float* lse0, float* lse1, cudaStream_t stream) {
    const HeadPlan h = head_plan(c.T, c.N, c.K);
    if (h.few) return head_few_forward(c, h, loss0, loss1, lse0, lse1, stream);
    const HeadWs w = head_ws_layout(h, false, c.T, c.K, c.top);
    HeadMaps maps;
    if (!head_encode(c, h, w, h.bn, &maps)) return SBN_ERR_CUDA;
    HeadRowsJob rows{};
    rows.loss0 = loss0; rows.loss1 = loss1; rows.lse0 = lse0; rows.lse1 = lse1;
    HeadLogitsParams p{};
    sbn_status st = launch_head_targets(c, w, &p.tg, stream);
    rows.tg = p.tg;
    if (st == SBN_OK && !h.words) st = launch_head_rows(c, w, rows, stream);
    if (st != SBN_OK) return st;
    const bool list = c.top != 0, dual = list && c.labels;
    if (!h.words) {
        p.count = reinterpret_cast<int*>(c.ws + w.count);
        p.row_src = reinterpret_cast<int*>(c.ws + w.row_src);
    }
    p.T = c.T; p.N = c.N; p.K = c.K;
    p.v0 = 0; p.v1 = c.N; p.bn = h.bn;
    p.c0 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K) / static_cast<double>(c.tau));
    p.c1 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K));
    p.part = reinterpret_cast<float2*>(c.ws + w.part);
    p.part1 = dual ? reinterpret_cast<float*>(c.ws + w.part1) : nullptr;
    p.z_ev = reinterpret_cast<float*>(c.ws + w.z_ev);
    p.parts = h.parts;
    p.skip_loads = g_test_break_waits;
    st = h.words ? launch_head_words<0>(maps, HeadWordsParams{p, words_stages(h.tokens), h.tokens, h.groups, h.word_pairs, nullptr, nullptr, HeadScale{}, 0}, list, dual, stream)
                 : launch_head_logits<0>(maps, p, list, dual, stream);
    if (st != SBN_OK) return st;
    return launch_head_losses(HeadLossJob{p.tg, p.count, p.row_src, c.T, c.N, p.part, p.part1, p.z_ev, static_cast<const uint16_t*>(c.x),
                                          static_cast<const uint16_t*>(c.head), c.K, h.parts, 1.0 / static_cast<double>(c.tau),
                                          head_logit_scale(c.K), loss0, loss1, lse0, lse1}, stream);
}

template <bool WIDE>
static sbn_status launch_head_grads(const HeadGradMaps& maps, const HeadGradParams& p, cudaStream_t stream) {
    using Loop = PairLoop<HeadGradsWork<WIDE>>;
    if (!ensure_dynamic_smem<head_grads_kernel<WIDE>>(Loop::kSmemBytes)) return SBN_ERR_CUDA;
    if (launch_kernel(head_grads_kernel<WIDE>, dim3(2 * kBackwardPairs), dim3(Loop::kThreads), Loop::kSmemBytes, stream, maps, p) != cudaSuccess)
        return SBN_ERR_CUDA;
    ++g_launch_count;
    return SBN_OK;
}

static sbn_status head_backward(const HeadCall& c, const float* lse0, const float* lse1, const float* g0, const float* g1, void* dx, void* dhead,
                                cudaStream_t stream) {
    const HeadPlan h = head_plan(c.T, c.N, c.K);
    if (h.few) return head_few_backward(c, h, lse0, lse1, g0, g1, dx, dhead, stream);
    const HeadWs w = head_ws_layout(h, true, c.T, c.K, c.top);
    const uint64_t k = static_cast<uint64_t>(c.K), t = static_cast<uint64_t>(c.T), grad_rows = static_cast<uint64_t>(h.grad_rows);
    HeadMaps maps;
    HeadGradMaps gm;
    if (!head_encode(c, h, w, h.bn_piece, &maps) || !encode_out(&maps.dz, c.ws + w.dz, true, h.piece, h.rows256, 1)) return SBN_ERR_CUDA;
    const uint32_t blocks = h.wide_grads ? 4 : 2;                       // of 64 columns, in a whole tile's box of B
    bool ok = encode_3d_bf16_blocks(&gm.aw, c.ws + w.dz, h.piece, h.rows256, 2) && encode_2d_bf16_sw128(&gm.ax, c.ws + w.dz, h.piece, h.rows256, h.piece, 128);
    for (int half = 0; ok && half < 2; ++half)
        ok = (h.words || encode_3d_bf16_blocks(&gm.bx[half], c.x, k, t, blocks >> half)) && encode_3d_bf16_blocks(&gm.bxc[half], c.ws + w.xc, k, h.rows64, blocks >> half);
    ok = ok && (!dx || encode_out(&gm.acc, c.ws + w.acc, false, k, grad_rows, h.slots));
    if (!ok) return SBN_ERR_CUDA;
    HeadRowsJob rows{};
    if (!h.words) rows.row_of = reinterpret_cast<int*>(c.ws + w.row_of);
    rows.scale = HeadScale{g0, g1, static_cast<float>(1.0 / static_cast<double>(c.tau)), reinterpret_cast<float*>(c.ws + w.scale)};
    HeadLogitsParams p{};
    p.scale = rows.scale.out;
    sbn_status st = launch_head_targets(c, w, &p.tg, stream);
    rows.tg = p.tg;
    if (st == SBN_OK && !h.words) st = launch_head_rows(c, w, rows, stream);
    if (st != SBN_OK) return st;
    const bool list = c.top != 0, dual = list && c.labels;
    if (!h.words) {
        p.count = reinterpret_cast<int*>(c.ws + w.count);
        p.row_src = reinterpret_cast<int*>(c.ws + w.row_src);
    }
    p.T = c.T; p.N = c.N; p.K = c.K;
    p.bn = h.bn_piece;
    p.c0 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K) / static_cast<double>(c.tau));
    p.c1 = static_cast<float>(1.4426950408889634 * head_logit_scale(c.K));
    p.inv_tau = static_cast<float>(1.0 / static_cast<double>(c.tau));
    p.lse0 = lse0; p.lse1 = lse1; p.g0 = g0; p.g1 = g1;
    p.skip_loads = g_test_break_waits;
    HeadGradParams q{};
    q.count = p.count;
    q.scale = p.scale;
    q.T = h.grad_rows; q.K = c.K;
    q.slot_stages = h.slot_stages;
    q.want_dx = dx != nullptr;
    q.want_dw = dhead != nullptr;
    q.skip_loads = g_test_break_waits;
    const int tiles_k = h.wide_grads ? (c.K + 511) / 512 : (c.K + 255) / 256;
    for (int v0 = 0; v0 < c.N; v0 += h.piece) {
        const int cols = std::min(h.piece, c.N - v0);
        p.v0 = v0; p.v1 = v0 + cols;
        st = h.words ? launch_head_words<1>(maps, HeadWordsParams{p, words_stages(h.tokens), h.tokens, h.groups, h.word_pairs, static_cast<const uint16_t*>(c.x), reinterpret_cast<uint16_t*>(c.ws + w.xc), rows.scale, h.rest},
                                            list, dual, stream)
                     : launch_head_logits<1>(maps, p, list, dual, stream);
        if (st != SBN_OK) return st;
        const char* w_rows = static_cast<const char*>(c.head) + static_cast<size_t>(v0) * c.K * 2;
        for (int half = 0; half < 2; ++half)
            if (!encode_3d_bf16_blocks(&gm.bw[half], w_rows, k, cols, blocks >> half)) return SBN_ERR_CUDA;
        const int all_stages = (cols + 63) / 64;
        q.cols = cols;
        if (dhead && !encode_out(&gm.dw, static_cast<uint16_t*>(dhead) + static_cast<size_t>(v0) * c.K, true, k, cols, 1)) return SBN_ERR_CUDA;
        q.add = v0 > 0;
        const int slices = (all_stages + h.slot_stages - 1) / h.slot_stages;     // fewer in a short last piece
        const int tiles[2] = {dhead ? (cols + 255) / 256 * tiles_k : 0, dx ? static_cast<int>(h.rows256 / 256) * tiles_k * slices : 0};
        const int stages[2] = {(h.grad_rows + 63) / 64, h.slot_stages};
        q.plan = plan_backward(tiles, stages, -1, 7.5);
        st = h.wide_grads ? launch_head_grads<true>(gm, q, stream) : launch_head_grads<false>(gm, q, stream);
        if (st != SBN_OK) return st;
    }
    return dx ? launch_head_dx(HeadDxJob{rows.row_of, reinterpret_cast<const float*>(c.ws + w.acc), h.slots, c.T, c.K, h.grad_rows, h.rest, p.scale, static_cast<uint16_t*>(dx)}, stream) : SBN_OK;
}

}  // namespace sbn
