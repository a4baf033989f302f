// The logits' tiles for up to 256 tokens: words on the lanes.  The head streams by once and is what such a call costs, so a tile
// is 256 words x the tokens there are (M = 256, N = the tokens up to a multiple of 32, half of them from either CTA of the pair):
// no row of the MMA is padding, and a stage brings 16 KB of words and no more tokens than there are.  With tokens on the
// lanes (head_gemm_tcgen05.cuh) 17 to 256 tokens cost the time of 256 rows per MMA: 2560 x 32000 took 46 to 60 us.  On single
// CTAs (128 words, every CTA with all tokens) the tokens' way from the L2 to the SMs was the limit: 226 tokens x 3712 x 41540 86 us.
// Where the words' tiles are too few to go round, the tokens are cut into groups as well.
//
// The epilogue turns 32 words x 32 tokens at a time around through shared memory, so that a thread owns a token there too
// (HeadRow); a token's maximum and sums lie in shared memory between tiles, per warp.  Tokens that nothing is asked of stay
// where they are: their column of the product reaches nobody (stats) or is replaced by zeros (grad), and the grad kernel
// leaves a copy of x with zeros in their rows for dW.
#pragma once

#include "head_gemm_tcgen05.cuh"

namespace sbn {

constexpr int kWordsTokens = 256;
// Up to this many tokens dz is kept in two bf16 parts, the second as further rows behind the first's (and x twice, one below the other).  The
// fewer the tokens, the fewer the entries that make a gradient, and the less their roundings average out: with one part 1.7 % of steps of up to
// 128 tokens had gradients 2.5e-3 to 3.7e-3 off in the 2-norm, where their own rounding is 1.7e-3; above that 0.2 % do, 2.6e-3 at most.  Both parts fit the
// one tile of 256 rows that dx has, so this costs 3 % (64 x 4096 x 131072 745 -> 770 us) to 8 % (128 x 2560 x 32000 146 -> 159 us) of a backward call.
constexpr int kWordsTwoParts = 128;
constexpr int kWordsSquare = 32 * 33;                                      // floats
constexpr int kWordsTurnBytes = 8 * kWordsSquare * 4;
constexpr int kWordsStateBytes = 8 * 3 * kWordsTokens * 4;                 // stats: [warp][m, s0, s1 or label][token]; grad: the warps' boxes
static_assert(kWordsTurnBytes % 1024 == 0 && kWordsStateBytes >= 8 * kWarpBoxBytes, "alignment and room of the boxes");

// What a CTA has per stage: 128 words, half the tokens.
__host__ __device__ constexpr int words_stage_bytes(int tokens) { return kPairLoopStageA + tokens / 2 * 128; }
// Few tokens leave room for more stages: it is the bytes under way that the words stream with.
constexpr int words_stages(int tokens) {
    const int room = (232448 - kBarrierBytes - kWordsTurnBytes - kWordsStateBytes) / words_stage_bytes(tokens);
    return room < 10 ? room : 10;
}
constexpr int words_smem_bytes(int tokens) { return words_stages(tokens) * words_stage_bytes(tokens) + kWordsTurnBytes + kWordsStateBytes + kBarrierBytes; }

struct HeadWordsParams {
    HeadLogitsParams p;           // rows are tokens: count, row_src, bn unused; parts = 8 x pairs
    int stages;
    int tokens, groups;           // tokens per tile (a multiple of 32), groups of them
    int pairs;
    const uint16_t* x;            // grad: copied to xc [T up to a multiple of 64][K]
    uint16_t* xc;
    HeadScale scale;              // grad
    int rest;                     // grad: rows of dz and xc from a token's to its second part's, 0: there is none
};

// REST: dz in two parts (grad).
template <int MODE, bool LIST, bool DUAL, bool REST>
struct HeadWordsWork {
    static constexpr bool kWide = false;
    static constexpr int kStages = 5, kStagingBytes = kWordsTurnBytes + kWordsStateBytes;    // (at 256 tokens)
    __device__ int stages() const { return wp.stages; }
    __device__ int stage_bytes() const { return words_stage_bytes(wp.tokens); }
    const HeadMaps& maps;
    const HeadWordsParams& wp;
    const HeadLogitsParams& p;
    int tiles_v;

    __device__ HeadWordsWork(const HeadMaps& m, const HeadWordsParams& q) : maps(m), wp(q), p(q.p) {}
    __device__ void start() { tiles_v = (p.v1 - p.v0 + 255) / 256; }

    struct Tile { int n0, t0, bn, k_stages; };                              // first word, first token, tokens
    struct Tiles {
        const HeadWordsWork& w;
        int i;
        __device__ Tiles(const HeadWordsWork& work, int pair) : w(work), i(pair) {}
        __device__ bool next(Tile& t) {
            if (i >= w.tiles_v * w.wp.groups) return false;
            t.n0 = w.p.v0 + i / w.wp.groups * 256;
            t.t0 = i % w.wp.groups * w.wp.tokens;
            t.bn = w.wp.tokens;
            t.k_stages = w.p.K >> 6;
            i += w.wp.pairs;
            return true;
        }
    };
    __device__ void load(const Tile& t, int ks, uint32_t rank, uint32_t st, uint32_t bar) const {
        tma_load_2d_pair(st, &maps.w, ks * 64, t.n0 + static_cast<int>(rank) * 128, bar);
        tma_load_2d_pair(st + kPairLoopStageA, &maps.x, ks * 64, t.t0 + static_cast<int>(rank) * (t.bn >> 1), bar);
    }
    __device__ uint32_t idesc(const Tile& t) const { return make_idesc_bf16_any(256, t.bn, false, false); }
    __device__ uint64_t a_step(const Tile&) const { return 32 >> 4; }
    __device__ uint64_t b_step(const Tile&) const { return 32 >> 4; }
    __device__ uint64_t a_desc(const Tile&, uint32_t s) const { return make_smem_desc(s, 16, 1024, kSwz128); }
    __device__ uint64_t b_desc(const Tile&, uint32_t s) const { return make_smem_desc(s, 16, 1024, kSwz128); }

    struct Epilogue {
        const HeadWordsWork& w;
        int rank, quarter, sub, lane;
        float* square;
        float* state;                                                       // stats: [m, s0, s1][token]; cross entropy has labels for s1
        uint32_t box;                                                       // grad
        float inv_scale;
        HeadRow<MODE, LIST, DUAL> row;

        __device__ Epilogue(const HeadWordsWork& work, int rk, int q, int sb, int ln, uint32_t staging) : w(work), rank(rk), quarter(q), sub(sb), lane(ln) {
            extern __shared__ uint8_t smem_raw[];
            uint8_t* mine = smem_raw + (staging - smem_u32(smem_raw));
            const int warp = sub * 4 + quarter;
            square = reinterpret_cast<float*>(mine) + warp * kWordsSquare;
            state = reinterpret_cast<float*>(mine + kWordsTurnBytes) + warp * 3 * kWordsTokens;
            box = staging + kWordsTurnBytes + static_cast<uint32_t>(warp * kWarpBoxBytes);
            inv_scale = 1.0f;
            const HeadLogitsParams& p = w.p;
            if constexpr (MODE == 0) {
                for (int t = lane; t < kWordsTokens; t += 32) {
                    state[t] = -INFINITY;
                    state[kWordsTokens + t] = state[2 * kWordsTokens + t] = 0.0f;
                    if constexpr (!LIST) {                                  // read here, where it waits for nothing
                        const bool there = t < p.T && (head_token_flags(p.tg, t, p.N) & kRowLabel);
                        state[2 * kWordsTokens + t] = __int_as_float(there ? static_cast<int>(p.tg.labels[t]) : kNoColumn);
                    }
                }
            } else {
                float largest = 0.0f;                                       // every warp for itself
                for (int t = lane; t < p.T; t += 32) largest = fmaxf(largest, head_scale_share(w.wp.scale, LIST, head_token_flags(p.tg, t, p.N), t));
                const float unit = head_scale_unit(warp_max(largest));
                inv_scale = 1.0f / unit;
                const int tid = static_cast<int>(threadIdx.x) - 64;
                if (blockIdx.x == 0 && tid == 0) {
                    w.wp.scale.out[0] = unit;
                    w.wp.scale.out[1] = inv_scale;
                }
                // x for dW, zeros in rows that nothing is asked of and behind the last token
                const int vecs = p.K >> 3, all = (p.T + 63) & ~63;
                for (int t = blockIdx.x; t < all; t += gridDim.x) {
                    const int flags = t < p.T ? head_token_flags(p.tg, t, p.N) : 0;
                    const bool there = (flags & (kRowDistill | kRowLabel)) != 0;
                    if (!LIST && tid == 0) report_bad(flags);
                    const uint4* from = reinterpret_cast<const uint4*>(w.wp.x + static_cast<size_t>(t) * p.K);
                    uint4* to = reinterpret_cast<uint4*>(w.wp.xc + static_cast<size_t>(t) * p.K);
                    for (int v = tid; v < vecs; v += 256) {
                        const uint4 value = there ? __ldg(from + v) : make_uint4(0u, 0u, 0u, 0u);
                        to[v] = value;
                        if constexpr (REST) to[static_cast<size_t>(w.wp.rest) * vecs + v] = value;
                    }
                }
            }
        }
        // A tile's chunks of 32 tokens; grad: dW contracts over whole stages of 64 rows, the last group's tile has zeros for them
        __device__ int chunks(const Tile& t) const {
            const int end = MODE == 0 ? w.p.T : (w.p.T + 63) & ~63;
            const bool last = t.t0 + t.bn >= w.p.T;
            return ((last ? end - t.t0 : t.bn) + 31) >> 5;
        }
        __device__ void begin(const Tile&) {}

        template <class Release>
        __device__ void run(const Tile& tile, uint32_t taddr, Release&& release) {
            const HeadLogitsParams& p = w.p;
            const int all = chunks(tile), n0 = tile.n0 + rank * 128 + quarter * 32;
            if (sub >= all) release();
#pragma unroll 1
            for (int c = sub; c < all; c += 2) {
                const int t = tile.t0 + c * 32 + lane;
                if constexpr (MODE == 0 && !LIST) {
                    const int label = __float_as_int(state[2 * kWordsTokens + t]);
                    row.begin(p, t, t, label != kNoColumn);
                    row.next_col = label >= n0 ? label : kNoColumn;
                } else {
                    const bool here = t < p.T && (head_token_flags(p.tg, t, p.N) & (kRowDistill | kRowLabel));
                    row.begin(p, t, here ? t : 0, here, inv_scale);
                    row.seek(p, n0);
                }
                uint32_t z[32];
                __syncwarp();
                // (behind the tile's tokens, but for less than 256 columns: whatever tensor memory holds, for nobody)
                tmem_ld_32x32b_x32(taddr + static_cast<uint32_t>(c * 32), z);
                tmem_ld_wait();
                if (c + 2 >= all) release();
#pragma unroll
                for (int q = 0; q < 32; ++q) square[q * 33 + lane] = __uint_as_float(z[q]);
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 32; ++q) z[q] = __float_as_uint(square[lane * 33 + q]);
                if constexpr (MODE == 0) {
                    const bool keep = t < p.T;
                    if (keep) {
                        row.m = state[t];
                        row.s0 = state[kWordsTokens + t];
                        if (DUAL) row.s1 = state[2 * kWordsTokens + t];
                    }
                    while (row.next_col < n0 + 32) {                        // a thread's token has its logits next to one another
                        p.z_ev[static_cast<size_t>(t) * p.tg.events + row.e] = square[lane * 33 + row.next_col - n0];
                        row.step(p);
                    }
                    __syncwarp();
                    row.stats(p, z, n0);
                    __syncwarp();
                    if (keep) {
                        state[t] = row.m;
                        state[kWordsTokens + t] = row.s0;
                        if (DUAL) state[2 * kWordsTokens + t] = row.s1;
                    }
                } else {
                    uint32_t o[16];
                    if constexpr (REST) {
                        uint32_t rest[16];
                        row.template grad<true>(p, z, n0, o, rest);
                        store_warp_box(box, lane, o, [&] { tma_store_2d(&w.maps.dz, n0 - p.v0, tile.t0 + c * 32, box); });
                        store_warp_box(box, lane, rest, [&] { tma_store_2d(&w.maps.dz, n0 - p.v0, w.wp.rest + tile.t0 + c * 32, box); });
                    } else {
                        row.grad(p, z, n0, o);
                        store_warp_box(box, lane, o, [&] { tma_store_2d(&w.maps.dz, n0 - p.v0, tile.t0 + c * 32, box); });
                    }
                }
            }
        }
        __device__ void finish() {
            const HeadLogitsParams& p = w.p;
            if constexpr (MODE == 1) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            } else {
                // this warp's tokens: every second chunk of every group
                const int part = (static_cast<int>(blockIdx.x) * 4) + quarter;
                for (int g = 0; g < w.wp.groups; ++g) {
                    const Tile t{0, g * w.wp.tokens, w.wp.tokens, 0};
                    for (int c = sub; c < chunks(t); c += 2) {
                        const int tok = t.t0 + c * 32 + lane;
                        if (tok >= p.T) continue;
                        row.begin(p, tok, tok, true);
                        row.m = state[tok];
                        row.s0 = state[kWordsTokens + tok];
                        if (DUAL) row.s1 = state[2 * kWordsTokens + tok];
                        row.store_part(p, part);
                    }
                }
            }
        }
    };
};

template <int MODE, bool LIST, bool DUAL, bool REST>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(320, 1)
head_words_kernel(const __grid_constant__ HeadMaps maps, const __grid_constant__ HeadWordsParams p) {
    pdl_launch_dependents();
    HeadWordsWork<MODE, LIST, DUAL, REST> work(maps, p);
    bf16_pair_loop(work, p.p.skip_loads != 0);
}

}  // namespace sbn
