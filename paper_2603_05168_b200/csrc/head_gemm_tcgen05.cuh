// The products at the output head, z = x W^T [T][N] (N = vocabulary), dx = dz W and dW = dz^T x, without z or dz ever being
// kept whole, on the CTA-pair loop of gemm_bf16_pair_loop.cuh:
//
//   head_logits_kernel<stats>   tiles of 256 rows x BN columns of z whose epilogue leaves, per row and half of a tile's columns,
//                               the maximum m and sum exp((z - m) / tau), and the logits at the row's targets
//   head_logits_kernel<grad>    the same tiles of one piece of the vocabulary (as many columns as the workspace holds):
//                               dz = g (exp(z / tau - lse) - target), rounded to bf16 into the piece
//   head_grads_kernel           both gradients of a piece in one launch: dW rows of the piece (contraction over the rows that
//                               count, bf16 out), and the piece's part of dx, added up in fp32
//
// Tokens are on the lanes of tensor memory, so an epilogue thread owns a token's row of the tile: its maximum, its sum and its
// targets need no exchange.  dz is rounded to bf16 because the tensor cores' operands are; sums are in fp32 throughout.  It is
// kept in units of the largest gradient of a loss (head_scale): with the mean's 1 / count everywhere, a target's p - 1 would
// else be rounded at an unlucky place of the binade in every row alike.
// Forward 2 T N K operations, a training step four times that (z is computed twice, it costs less than keeping it).
#pragma once

#include "gemm_bf16_pair_loop.cuh"
#include "head_rows.cuh"

namespace sbn {

__device__ __forceinline__ float ex2_approx(float v) {        // relative error 2^-22
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ void st_shared_16(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int c0, int c1, int c2, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* map, int c0, int c1, int c2, uint32_t src) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(src) : "memory");
}

// 32 rows x 64 bytes of a warp (lane = row) through kWarpBoxBytes of shared memory of its own: the 16-byte pieces q of a row at
// q ^ (row / 2 % 4), as the 64-byte swizzle has them; store() issues the TMA store.  Waits until no more than
// PENDING stores of the warp are still to be read out: one box, or two in turn.
constexpr int kWarpBoxBytes = 2048;
template <int PENDING = 0, class Store>
__device__ __forceinline__ void store_warp_box(uint32_t box, int lane, const uint32_t (&v)[16], Store&& store) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
    const uint32_t to = box + static_cast<uint32_t>(lane * 64), x = static_cast<uint32_t>(lane >> 1) & 3u;
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) st_shared_16(to + ((q ^ x) << 4), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        store();
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ void tmem_ld_32x32b_x1(uint32_t taddr, uint32_t& r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
}

// The tensor cores cut a running sum off after every 16 columns instead of rounding it, so a sum whose terms change sign comes out
// too small: by K 2^-30 of itself on average (0.8 to 1.1 times that at K = 256 to 2^20; the single logit is off by half of it
// more or less).  Taken back where logits are used, at no cost: losses of 2048 tokens x 2560 4.7e-7 off -> 0.7e-7.  Other sums it
// does not fit, either way by as little: one that fits 24 bits was right and is K 2^-30 too large (2.4e-6 of the logit at 2560 columns),
// one whose terms are all of a sign stays 2 to 5 times that too small.
static inline double head_logit_scale(int K) { return 1.0 + K * 0x1p-30; }

struct HeadMaps {
    CUtensorMap x, xc;            // K-major: the tokens' rows, or the rows that count moved together
    CUtensorMap w;                // K-major, BN / 2 rows per box
    CUtensorMap dz;               // grad: [T up to a multiple of 256][columns of a piece], stored in boxes of 32 rows x 64 bytes
};
struct HeadLogitsParams {
    HeadTargets tg;
    const int* count;
    const int* row_src;
    int T, N, K;
    int v0, v1;                   // columns of z: the whole vocabulary, or a piece
    int bn;
    float c0, c1;                 // log2(e) / tau and log2(e), times head_logit_scale
    // stats
    float2* part;                 // [rows][parts]
    float* part1;                 // [rows][parts], sums at temperature 1 (with labels)
    float* z_ev;                  // [rows][events]: logits at the targets
    int parts;
    // grad
    const float *lse0, *lse1;     // per token
    const float *g0, *g1;         // gradients of the two losses per token (g1: label beside a teacher)
    float inv_tau;
    const float* scale;           // see HeadScale
    int skip_loads;
};

// MODE 0 stats, 1 grad.  LIST: targets are sorted events (distillation), else the label alone.  DUAL: the label's loss at
// temperature 1 beside the teacher's.
//
// What a thread does with the logits of its row, 32 neighbouring columns at a time in ascending order.
template <int MODE, bool LIST, bool DUAL>
struct HeadRow {
    int r, t;                     // row of the products, its token
    bool here;                    // something is asked of it
    int next_col, e;              // the next target at or behind the current column
    float l0, l1, g0, g1;         // grad: -lse log2(e) and gradient per loss
    float m, s0, s1;              // stats

    static constexpr float kLog2e = 1.4426950408889634f;

    // Row r with token t; `asked` says whether anything is asked of it.
    __device__ void begin(const HeadLogitsParams& p, int row, int token, bool asked, float inv_scale = 1.0f) {
        r = row;
        t = token;
        here = asked;
        next_col = kNoColumn;
        e = 0;
        m = l0 = l1 = -INFINITY;
        s0 = s1 = g0 = g1 = 0.0f;
        if constexpr (MODE == 1) {
            if (!here) return;
            const int flags = LIST ? p.tg.flags[t] : kRowDistill;
            if (flags & kRowDistill) {
                l0 = -p.lse0[t] * kLog2e;
                g0 = p.g0[t] * p.inv_tau * inv_scale;
            }
            if (DUAL && (flags & kRowLabel)) {
                l1 = -p.lse1[t] * kLog2e;
                g1 = p.g1[t] * inv_scale;
            }
        }
    }
    __device__ const int* list(const HeadLogitsParams& p) const { return p.tg.ev_col + static_cast<size_t>(t) * p.tg.events; }
    // To the first target at or behind column n.
    __device__ void seek(const HeadLogitsParams& p, int n) {
        next_col = kNoColumn;
        if (!here) return;
        if constexpr (LIST) {
            const int* col = list(p);
            int lo = 0, hi = p.tg.events;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (col[mid] < n) lo = mid + 1; else hi = mid;
            }
            e = lo;
            if (e < p.tg.events) next_col = col[e];
        } else {
            const int label = static_cast<int>(p.tg.labels[t]);
            if (label >= n) next_col = label;
        }
    }
    __device__ void step(const HeadLogitsParams& p) {
        if constexpr (LIST) {
            ++e;
            next_col = e < p.tg.events ? list(p)[e] : kNoColumn;
        } else {
            next_col = kNoColumn;
        }
    }

    // Writes down the row's logits at its targets among columns n .. n + 31; at(q) gives every lane of the warp its logit of column
    // n + q.  The whole warp takes part (picking a register by an index of the lane's own would put all 32 into local memory:
    // 1 us per 32 columns).  A row has a handful of targets in the whole vocabulary, the label's among them: head_losses_kernel
    // takes its term out of the sum.
    template <class At>
    __device__ void note_targets(const HeadLogitsParams& p, int n, At&& at) {
        while (next_col < n) step(p);
        for (uint32_t who; (who = __ballot_sync(0xFFFFFFFFu, next_col < n + 32)) != 0u;) {
            const int q = __shfl_sync(0xFFFFFFFFu, next_col - n, __ffs(who) - 1);
            const float v = at(q);
            if (next_col - n == q) {
                p.z_ev[static_cast<size_t>(r) * p.tg.events + e] = v;
                step(p);
            }
        }
    }
    // Columns n .. n + 31.
    __device__ void stats(const HeadLogitsParams& p, uint32_t (&z)[32], int n) {
        if (n >= p.N) return;
        if (n + 32 > p.N) {                            // behind the vocabulary: nothing
#pragma unroll
            for (int q = 0; q < 32; ++q) z[q] = n + q < p.N ? z[q] : 0xFF800000u;
        }
        float mc[4] = {m, m, m, m};                    // four chains: a chain of 32 would wait for itself
#pragma unroll
        for (int q = 0; q < 32; ++q) mc[q & 3] = fmaxf(mc[q & 3], __uint_as_float(z[q]));
        const float m_new = fmaxf(fmaxf(mc[0], mc[1]), fmaxf(mc[2], mc[3]));
        float a0[4] = {s0 * ex2_approx((m - m_new) * p.c0), 0.0f, 0.0f, 0.0f}, a1[4] = {};
        if (DUAL) a1[0] = s1 * ex2_approx((m - m_new) * p.c1);
        m = m_new;
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            const float d = __uint_as_float(z[q]) - m;      // the difference first: exact where it matters
            a0[q & 3] += ex2_approx(d * p.c0);
            if (DUAL) a1[q & 3] += ex2_approx(d * p.c1);
        }
        s0 = (a0[0] + a0[1]) + (a0[2] + a0[3]);
        if (DUAL) s1 = (a1[0] + a1[1]) + (a1[2] + a1[3]);
    }
    __device__ void store_part(const HeadLogitsParams& p, int part) const {
        const size_t at = static_cast<size_t>(r) * p.parts + part;
        p.part[at] = make_float2(m, s0);
        if (DUAL) p.part1[at] = s1;
    }

    // Columns n .. n + 31 of dz in bf16, zeros in rows that nothing is asked of and behind the vocabulary; SPLIT: and what bf16 leaves off,
    // in bf16 again.
    template <bool SPLIT = false>
    __device__ void grad(const HeadLogitsParams& p, const uint32_t (&z)[32], int n, uint32_t (&o)[16], uint32_t* rest = nullptr) {
        while (next_col < n) step(p);
        float v[32];
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            v[q] = ex2_approx(fmaf(__uint_as_float(z[q]), p.c0, l0)) * g0;
            if (DUAL) v[q] = fmaf(ex2_approx(fmaf(__uint_as_float(z[q]), p.c1, l1)), g1, v[q]);
        }
        while (next_col < n + 32) {
            float off = g0;
            if constexpr (LIST) {
                const float q = p.tg.ev_w[static_cast<size_t>(t) * p.tg.events + e];
                off = q < 0.0f ? g1 : q * g0;
            }
#pragma unroll
            for (int q = 0; q < 32; ++q) v[q] -= next_col - n == q ? off : 0.0f;
            step(p);
        }
        if (!here || n + 32 > p.N) {
#pragma unroll
            for (int q = 0; q < 32; ++q) v[q] = here && n + q < p.N ? v[q] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 16; ++q) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[q]) : "f"(v[2 * q + 1]), "f"(v[2 * q]));
        if constexpr (SPLIT) {
#pragma unroll
            for (int q = 0; q < 16; ++q)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(rest[q]) : "f"(v[2 * q + 1] - bf16hi_to_f32(o[q])), "f"(v[2 * q] - bf16lo_to_f32(o[q])));
        }
    }
};

template <int MODE, bool LIST, bool DUAL>
struct HeadLogitsWork {
    static constexpr bool kWide = false;
    static constexpr int kStages = MODE == 0 ? 7 : 6, kStagingBytes = MODE == 0 ? 0 : 8 * kWarpBoxBytes;
    __device__ static constexpr int stages() { return kStages; }
    __device__ static constexpr int stage_bytes() { return PairLoop<HeadLogitsWork>::kStageBytes; }
    const HeadMaps& maps;
    const HeadLogitsParams& p;
    int rows, tiles_m, tiles_v;
    float inv_scale;
    bool moved;

    __device__ HeadLogitsWork(const HeadMaps& m, const HeadLogitsParams& q) : maps(m), p(q) {}
    __device__ void start() {
        rows = *p.count;
        inv_scale = MODE == 1 ? p.scale[1] : 1.0f;
        moved = rows < p.T;
        tiles_m = (max(rows, 1) + 255) / 256;              // no row counts: one tile of zeros, which dW then contracts over
        tiles_v = (p.v1 - p.v0 + p.bn - 1) / p.bn;
    }

    struct Tile { int m0, n0, bn, k_stages; };
    // Row tiles fastest, in groups of 16 (a group's rows stay in the L2 while the vocabulary streams by once).
    struct Tiles {
        const HeadLogitsWork& w;
        long long i;
        long long all;
        __device__ Tiles(const HeadLogitsWork& work, int pair) : w(work), i(pair), all(static_cast<long long>(work.tiles_m) * work.tiles_v) {}
        __device__ bool next(Tile& t) {
            if (i >= all) return false;
            const int group = static_cast<int>(i / (16ll * w.tiles_v));
            const int in_group = min(16, w.tiles_m - 16 * group);
            const int rem = static_cast<int>(i - 16ll * group * w.tiles_v);
            t.m0 = (16 * group + rem % in_group) * 256;
            t.n0 = w.p.v0 + (rem / in_group) * w.p.bn;
            t.bn = w.p.bn;
            t.k_stages = w.p.K >> 6;
            i += kBackwardPairs;
            return true;
        }
    };

    __device__ void load(const Tile& t, int ks, uint32_t rank, uint32_t st, uint32_t bar) const {
        tma_load_2d_pair(st, moved ? &maps.xc : &maps.x, ks * 64, t.m0 + static_cast<int>(rank) * 128, bar);
        tma_load_2d_pair(st + kPairLoopStageA, &maps.w, ks * 64, t.n0 + static_cast<int>(rank) * (t.bn >> 1), bar);
    }
    __device__ uint32_t idesc(const Tile& t) const { return make_idesc_bf16_any(256, t.bn, false, false); }
    __device__ uint64_t a_step(const Tile&) const { return 32 >> 4; }
    __device__ uint64_t b_step(const Tile&) const { return 32 >> 4; }
    __device__ uint64_t a_desc(const Tile&, uint32_t s) const { return make_smem_desc(s, 16, 1024, kSwz128); }
    __device__ uint64_t b_desc(const Tile&, uint32_t s) const { return make_smem_desc(s, 16, 1024, kSwz128); }

    struct Epilogue {
        const HeadLogitsWork& w;
        int rank, quarter, sub, lane;
        uint32_t box;
        HeadRow<MODE, LIST, DUAL> row;

        __device__ Epilogue(const HeadLogitsWork& work, int rk, int q, int sb, int ln, uint32_t staging)
            : w(work), rank(rk), quarter(q), sub(sb), lane(ln), box(staging + static_cast<uint32_t>((sb * 4 + q) * kWarpBoxBytes)) {}
        __device__ void begin(const Tile& tile) {
            const int r = tile.m0 + rank * 128 + quarter * 32 + lane;
            const bool here = r < w.rows;
            row.begin(w.p, r, here ? w.p.row_src[r] : 0, here, w.inv_scale);
            row.seek(w.p, tile.n0);
        }
        template <class Release>
        __device__ void run(const Tile& tile, uint32_t taddr, Release&& release) {
            const int chunks = tile.bn >> 5;
            const int first_row = tile.m0 + rank * 128 + quarter * 32;
            // rows that nobody reads: behind the last that counts (grad: behind the last stage that dW reads)
            if (first_row >= (MODE == 0 ? w.rows : ((max(w.rows, 1) + 63) & ~63))) {
                release();
                return;
            }
#pragma unroll 1
            for (int c = sub; c < chunks; c += 2) {
                uint32_t z[32];
                __syncwarp();                              // the lanes may have parted over their targets
                tmem_ld_32x32b_x32(taddr + static_cast<uint32_t>(c * 32), z);
                tmem_ld_wait();
                const int n = tile.n0 + c * 32;
                if constexpr (MODE == 0)
                    row.note_targets(w.p, n, [&](int q) {
                        uint32_t v;
                        tmem_ld_32x32b_x1(taddr + static_cast<uint32_t>(c * 32 + q), v);
                        tmem_ld_wait();
                        return __uint_as_float(v);
                    });
                if (c + 2 >= chunks) release();
                if constexpr (MODE == 0) {
                    row.stats(w.p, z, n);
                } else {
                    uint32_t o[16];
                    row.grad(w.p, z, n, o);
                    store_warp_box(box, lane, o, [&] { tma_store_2d(&w.maps.dz, n - w.p.v0, first_row, box); });
                }
            }
            if (MODE == 0 && row.here) row.store_part(w.p, 2 * ((tile.n0 - w.p.v0) / tile.bn) + sub);
        }
        __device__ void finish() {
            if (MODE == 1 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
    };
};

template <int MODE, bool LIST, bool DUAL>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(320, 1)
head_logits_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadLogitsParams p) {
    pdl_launch_dependents();
    HeadLogitsWork<MODE, LIST, DUAL> work(maps, p);
    bf16_pair_loop(work, p.skip_loads != 0);
}

// ---- gradients of a piece --------------------------------------------------------------------------
// dw, acc: how results leave, in boxes of 32 rows x 64 bytes.
struct HeadGradMaps {
    CUtensorMap aw;               // dz piece for dW: MN-major, two blocks of 64 columns
    CUtensorMap ax;               // dz piece for dx: K-major
    CUtensorMap bx[2], bxc[2];    // x, or the rows that count moved together: MN-major, whole and half tiles
    CUtensorMap bw[2];            // the piece's rows of W
    CUtensorMap dw;               // [cols][K] bf16
    CUtensorMap acc;              // [slots][T][K] fp32
};
struct HeadGradParams {
    const float* scale;           // dW leaves times this (HeadScale)
    const int* count;             // null: all rows, zeros in place of those left out (`moved` rows)
    int T, K;
    int cols;                     // vocabulary rows of the piece
    int slot_stages;              // dx's contraction is cut into slices of that many stages, each with a slot of its own
    int add;                      // not the first piece: add to acc
    int want_dx, want_dw;
    BackwardPlan plan;            // part 0: dW, part 1: dx (tile index = slice * tiles of dx + tile)
    int skip_loads;
};

template <bool WIDE>
struct HeadGradsWork {
    static constexpr bool kWide = WIDE;
    static constexpr int kStages = WIDE ? 4 : 6, kStagingBytes = 16 * kWarpBoxBytes, kTileCols = WIDE ? 512 : 256;
    __device__ static constexpr int stages() { return kStages; }
    __device__ static constexpr int stage_bytes() { return PairLoop<HeadGradsWork>::kStageBytes; }
    const HeadGradMaps& maps;
    const HeadGradParams& p;
    int rows;
    float scale;
    bool moved;

    __device__ HeadGradsWork(const HeadGradMaps& m, const HeadGradParams& q) : maps(m), p(q) {}
    __device__ void start() {
        rows = p.count != nullptr ? *p.count : p.T;
        scale = *p.scale;
        moved = p.count == nullptr || rows < p.T;
        if (fewer_rows()) share();
    }
    __device__ bool fewer_rows() const { return p.count != nullptr && rows < p.T; }
    __device__ int tiles_m() const { return (max(rows, 1) + 255) / 256; }

    // With rows left out (the count is known here only): dx's tiles, which are long, go round; dW's go to the pairs with one tile of dx
    // less first (`most` pairs have one more than the others), as many as are as long, then round.
    int dx_all, most, dw_each, dw_extra, dw_left;
    __device__ void share() {
        const int tiles_n = (p.K + kTileCols - 1) / kTileCols;
        const int slices = p.want_dx ? ((p.cols + 63) / 64 + p.slot_stages - 1) / p.slot_stages : 0;
        const int dw_all = p.want_dw ? (p.cols + 255) / 256 * tiles_n : 0;
        dx_all = tiles_m() * tiles_n * slices;
        most = dx_all % kBackwardPairs;
        const int others = kBackwardPairs - most;
        // stages of a tile, with its turnaround; a tile of dW takes as long as it takes to write
        const float dx_cost = static_cast<float>(p.slot_stages) + 3.0f, dw_cost = fmaxf(static_cast<float>((rows + 63) / 64), 7.5f) + 3.0f;
        const float each = (static_cast<float>(dw_all) - (most != 0 ? others * dx_cost / dw_cost : 0.0f)) / kBackwardPairs;
        float best = INFINITY;
        for (int up = 0; up < 2; ++up) {                // the even share, rounded down or up: whichever ends sooner
            const int n = min(max(0, static_cast<int>(floorf(each)) + up), dw_all / kBackwardPairs);
            const int rest = dw_all - n * kBackwardPairs, extra = rest / others, left = rest % others;
            const float end = fmaxf((n + extra + (left != 0 ? 1 : 0)) * dw_cost, most != 0 ? dx_cost + n * dw_cost : 0.0f);
            if (end < best) {
                best = end;
                dw_each = n;
                dw_extra = extra;
                dw_left = left;
            }
        }
    }
    __device__ int dx_of(int pair) const { return dx_all / kBackwardPairs + (pair < most ? 1 : 0); }
    // The i-th tile of dW of a pair, -1: no more.
    __device__ int dw_of(int pair, int i) const {
        if (i < dw_each) return i * kBackwardPairs + pair;
        const int at = i - dw_each, who = pair - most, others = kBackwardPairs - most;
        if (who < 0 || at > dw_extra || (at == dw_extra && who >= dw_left)) return -1;
        return dw_each * kBackwardPairs + at * others + who;
    }

    struct Tile { int part, m0, n0, bn, k_stages, k_first, slot; };
    struct Tiles {
        const HeadGradsWork& w;
        int pair, g, i;
        __device__ Tiles(const HeadGradsWork& work, int pr) : w(work), pair(pr), g(0), i(0) {}
        // Entry u of a part: a whole tile, or a half of tile first + u / 2.
        __device__ void set(Tile& t, int part, int u, bool half, int first) const {
            const HeadGradParams& p = w.p;
            const int tiles_n = (p.K + kTileCols - 1) / kTileCols;
            t.part = part;
            t.bn = half ? kTileCols / 2 : kTileCols;
            int tile = half ? first + (u >> 1) : u;
            t.slot = 0;
            t.k_first = 0;
            if (part == 0) {
                // words' tiles next to one another, so that their dz comes from memory once (x stays in the L2)
                t.k_stages = (max(w.rows, 1) + 63) / 64;
                t.m0 = tile / tiles_n * 256;
                t.n0 = tile % tiles_n * kTileCols;
            } else {
                // all tiles run along the vocabulary side by side
                const int tiles_m = w.tiles_m(), tiles = tiles_m * tiles_n;
                t.slot = tile / tiles;
                tile -= t.slot * tiles;
                t.k_first = t.slot * p.slot_stages;
                t.k_stages = min(p.slot_stages, (p.cols + 63) / 64 - t.k_first);
                t.m0 = tile % tiles_m * 256;
                t.n0 = tile / tiles_m * kTileCols;
            }
            if (half) t.n0 += (u & 1) * (kTileCols / 2);
        }
        __device__ bool next(Tile& t) {
            const HeadGradParams& p = w.p;
            if (w.fewer_rows()) {                       // the host's plan is for all rows
                if (i < w.dx_of(pair)) {
                    set(t, 1, i * kBackwardPairs + pair, false, 0);
                } else {
                    const int u = w.dw_of(pair, i - w.dx_of(pair));
                    if (u < 0) return false;
                    set(t, 0, u, false, 0);
                }
                ++i;
                return true;
            }
            for (; g < p.plan.segments; ++g, i = 0) {
                const BackwardSegment& sg = p.plan.seg[g];
                if (i < sg.count(pair)) {
                    set(t, sg.part, sg.index(pair, i++), sg.half != 0, sg.first_tile);
                    return true;
                }
            }
            return false;
        }
    };

    __device__ void load(const Tile& t, int ks, uint32_t rank, uint32_t st, uint32_t bar) const {
        const int m0 = t.m0 + static_cast<int>(rank) * 128, n0 = t.n0 + static_cast<int>(rank) * (t.bn >> 1);
        const int half = t.bn < kTileCols, k = (t.k_first + ks) * 64;
        if (t.part == 0) tma_load_3d_pair(st, &maps.aw, 0, k, m0 >> 6, bar);
        else tma_load_2d_pair(st, &maps.ax, k, m0, bar);
        const CUtensorMap* b = t.part == 1 ? &maps.bw[half] : (moved ? &maps.bxc[half] : &maps.bx[half]);
        tma_load_3d_pair(st + kPairLoopStageA, b, 0, k, n0 >> 6, bar);
    }
    // K = 16 elements per instruction: 16 rows of an MN-major operand, 32 B along a row of a K-major one
    __device__ uint32_t idesc(const Tile& t) const { return make_idesc_bf16_any(256, WIDE ? 256 : t.bn, t.part == 0, true); }
    __device__ uint64_t a_step(const Tile& t) const { return t.part == 0 ? (2048 >> 4) : (32 >> 4); }
    __device__ uint64_t b_step(const Tile&) const { return 2048 >> 4; }
    __device__ uint64_t a_desc(const Tile& t, uint32_t s) const { return make_smem_desc(s, t.part == 0 ? 8192 : 16, 1024, kSwz128); }
    __device__ uint64_t b_desc(const Tile&, uint32_t s) const { return make_smem_desc(s, 8192, 1024, kSwz128); }

    // Results go out through shared memory and TMA stores, which also clip what lies outside: every warp has 2 KB of its own (narrow
    // tiles: twice) and stores boxes of 32 rows x 64 bytes.  Stored by the threads themselves, a row each, every 16 bytes were a
    // transaction of their own: 4 us per fp32 tile.
    struct Epilogue {
        const HeadGradsWork& w;
        int rank, quarter, parity, lane;                    // parity: `sub` of the loop (narrow: even or odd chunks)
        uint32_t staging;
        __device__ Epilogue(const HeadGradsWork& work, int rk, int q, int sub, int ln, uint32_t st)
            : w(work), rank(rk), quarter(q), parity(sub), lane(ln), staging(st + static_cast<uint32_t>((sub * 4 + q) * kWarpBoxBytes)) {}
        __device__ void begin(const Tile&) {}

        template <class Release>
        __device__ void run(const Tile& t, uint32_t taddr, Release&& release) {
            if constexpr (WIDE) run_wide(t, taddr, release);
            else run_narrow(t, taddr, release);
        }

        template <class Release>
        __device__ void run_wide(const Tile& t, uint32_t taddr, Release&& release) {
            const HeadGradParams& p = w.p;
            const int m = t.m0 + rank * 128 + quarter * 32;
            const int n0 = t.n0 + (t.bn == 512 ? 128 * (parity >> 1) + 256 * (parity & 1) : 128 * parity);
            if (m >= (t.part == 0 ? p.cols : w.rows) || n0 >= p.K || 128 * parity >= t.bn) {       // K % 128 == 0: the warp's columns are in or out as a whole
                release();
                return;
            }
            taddr += static_cast<uint32_t>(128 * parity);
            if (t.part == 0) {
                // all 128 columns into registers, halved in size, before anything is stored: the next tile's MMAs wait for this
                uint32_t o[4][16];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t v[16];
                    tmem_ld_32x32b_x16(taddr + static_cast<uint32_t>(c * 16), v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;"
                            : "=r"(o[c >> 1][8 * (c & 1) + i]) : "f"(__uint_as_float(v[2 * i + 1]) * w.scale), "f"(__uint_as_float(v[2 * i]) * w.scale));
                }
                release();
#pragma unroll
                for (int c = 0; c < 4; ++c) store_warp_box(staging, lane, o[c], [&] { tma_store_2d(&w.maps.dw, n0 + c * 32, m, staging); });
                return;
            }
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
                uint32_t v[16];
                __syncwarp();
                tmem_ld_32x32b_x16(taddr + static_cast<uint32_t>(c * 16), v);
                tmem_ld_wait();
                if (c == 7) release();
                store_warp_box(staging, lane, v, [&] { store_sums(t, n0 + c * 16, m, staging); });
            }
        }

        template <class Release>
        __device__ void run_narrow(const Tile& t, uint32_t taddr, Release&& release) {
            const HeadGradParams& p = w.p;
            const int m = t.m0 + rank * 128 + quarter * 32;
            const int chunks = min(t.bn, p.K - t.n0) >> 5;          // K % 128 == 0
            if (m >= (t.part == 0 ? p.cols : w.rows) || parity >= chunks) {
                release();
                return;
            }
#pragma unroll 1
            for (int c = parity; c < chunks; c += 2) {
                uint32_t v[32];
                __syncwarp();
                tmem_ld_32x32b_x32(taddr + static_cast<uint32_t>(c * 32), v);
                tmem_ld_wait();
                if (c + 2 >= chunks) release();
                const int n = t.n0 + c * 32;
                uint32_t o[16];
                if (t.part == 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(__uint_as_float(v[2 * i + 1]) * w.scale), "f"(__uint_as_float(v[2 * i]) * w.scale));
                    const uint32_t box = staging + static_cast<uint32_t>(((c >> 1) & 1) * 8 * kWarpBoxBytes);
                    store_warp_box<1>(box, lane, o, [&] { tma_store_2d(&w.maps.dw, n, m, box); });
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = v[16 * h + i];
                        const uint32_t box = staging + static_cast<uint32_t>(h * 8 * kWarpBoxBytes);
                        store_warp_box<1>(box, lane, o, [&] { store_sums(t, n + 16 * h, m, box); });
                    }
                }
            }
        }
        // One tile of a launch adds to an element, and launches follow one another: the sum's order is fixed
        __device__ void store_sums(const Tile& t, int n, int m, uint32_t box) const {
            if (w.p.add) tma_add_3d(&w.maps.acc, n, m, t.slot, box);
            else tma_store_3d(&w.maps.acc, n, m, t.slot, box);
        }
        __device__ void finish() {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
    };
};

template <bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WIDE ? 576 : 320, 1)
head_grads_kernel(const __grid_constant__ HeadGradMaps maps, const __grid_constant__ HeadGradParams p) {
    pdl_launch_dependents();
    HeadGradsWork<WIDE> work(maps, p);
    bf16_pair_loop(work, p.skip_loads != 0);
}

}  // namespace sbn
