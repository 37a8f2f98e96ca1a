// iso_attn_grad.cu -- attention's gradients on the fifth-generation tensor cores
// (bfloat16, head dimensions up to 128).
//
// The weights are formed again from lse, and both kernels own what they write, so
// there are no atomics and no binary32 gradients in memory; that takes seven products of
// 128 x 128 x dim a pair of tiles instead of five.
//   grad_kv   128 keys: over the query tiles (and query heads) that see them
//               S^T = K Q^T       P^T = exp2(c S^T - lse2)      dV += P^T dO
//               dP^T = V dO^T     dS^T = P^T (dP^T - delta)     dK += dS^T Q
//             Keys are rows, so that P^T and dS^T, rounded to bf16, go back to
//             tensor memory over the scores they came from and are the A operands of the
//             second products as they are; Q and dO serve both as rows to contract
//             along and as rows to contract over.  Two warps issue products, dV(i)
//             S(i+1) the one and dK(i) dP(i+1) the other: while the warps form P(i+1)
//             the second pair runs, and while they form dS(i+1) the first, with one buffer each
//             for scores and dP.  (One warp for both waited for either's turn: 1312
//             against 1160 us.)
//   grad_q    128 queries: over the key tiles that they see
//               S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//             with two buffers of scores; dS lies over its scores.
// Tensor memory is full in both (4 x 128 columns).  Eight warps compute, four on each
// GR_COLS columns of a tile; one warp copies, two issue products, and in grad_kv
// one more brings lse and delta, which are per column there.
// Measured: 8192 tokens, 28 heads over 4 of 128, causal, 1.03 - 1.11 ms (1.09 - 1.17
// PFLOP/s of the five products, 7/5 of that issued); tensor pipe 66 % active.  What
// bounds it is a step's chain: 300 - 700 clocks of waiting for its products, 1300 -
// 1900 of forming weights and gradients, against 1536 (grad_q) and 2048 of products.
#include "iso_attn.cuh"
#include "iso_attn_simt.cuh"
#include "iso_attn_tc.cuh"
#include "iso_tc.cuh"

#include <algorithm>
#include <cmath>

namespace iso {
namespace {

using namespace tc;

constexpr int GR_COMPUTE = 8;            // warps that compute, four on each GR_COLS columns of a tile
constexpr int GR_COLS = 64;
constexpr int GR_THREADS = (GR_COMPUTE + 4) * 32;
constexpr int KV_Q_STAGES = 3, KV_DO_STAGES = 2, Q_K_STAGES = 3, Q_V_STAGES = 2;

// the plan's estimates, in steps of dk and dv (1.45 us): a step of dq, a CTA's start and
// end, a join's launch, and the bytes that the card moves in one
constexpr double GR_Q_STEP = 0.72, GR_ITEM_STEPS = 6.0, GR_JOIN_STEPS = 1.5, GR_STEP_BYTES = 6.4e6;

struct GradMaps {
    CUtensorMap q, k, v, dout;
};

template <int DP>
struct GradTile {
    static constexpr int TILE = DP / BOX * BOX_BYTES;
    static constexpr int KV_SMEM = 1024 + (2 + KV_Q_STAGES + KV_DO_STAGES) * TILE + 2 * ROWS * 4 + 256;
    static constexpr int Q_SMEM = 1024 + (2 + Q_K_STAGES + Q_V_STAGES) * TILE + 256;
    static_assert(KV_SMEM <= 232448 && Q_SMEM <= 232448, "shared memory of one CTA");
    static_assert(sa_smem<DP>(4, 2) <= (2 + KV_Q_STAGES + KV_DO_STAGES) * TILE + 2 * ROWS * 4 &&
                  sa_smem<DP>(4, 1) <= (2 + Q_K_STAGES + Q_V_STAGES) * TILE, "the rows done over fit where the tiles were");
};

// The weights of COLS columns of this thread's row, p = exp2(c s - lse2), with the
// columns outside [from, to) 0 in a masked tile; neg_lse2(j): -lse2 of columns 2 j, 2 j + 1
template <bool MASKED, int COLS, typename L>
__device__ __forceinline__ void weights(const float (&s)[COLS], uint64_t (&p)[COLS / 2], uint64_t c, int from, int to, L neg_lse2) {
#pragma unroll
    for (int j = 0; j < COLS / 2; ++j) {
        float x, y;
        parts_of(fma2(pair_of(s[2 * j], s[2 * j + 1]), c, neg_lse2(j)), x, y);
        x = ex2(x);
        y = ex2(y);
        if (MASKED && !(2 * j >= from && 2 * j < to)) x = 0.0f;
        if (MASKED && !(2 * j + 1 >= from && 2 * j + 1 < to)) y = 0.0f;
        p[j] = pair_of(x, y);
    }
}
// dS = P (dP - delta) as bf16; what is not seen is 0 whatever dP is there
template <bool MASKED, int COLS, typename L>
__device__ __forceinline__ void score_grads(const float (&d)[COLS], const uint64_t (&p)[COLS / 2], uint32_t (&w)[COLS / 2], int from, int to,
                                            L neg_delta) {
#pragma unroll
    for (int j = 0; j < COLS / 2; ++j) {
        float x, y;
        parts_of(mul2(add2(pair_of(d[2 * j], d[2 * j + 1]), neg_delta(j)), p[j]), x, y);
        if (MASKED && !(2 * j >= from && 2 * j < to)) x = 0.0f;
        if (MASKED && !(2 * j + 1 >= from && 2 * j + 1 < to)) y = 0.0f;
        w[j] = f32_to_bf16x2(x, y);
    }
}
// COLS columns of this thread's row
template <int COLS>
__device__ __forceinline__ void load_cols(uint32_t at, float (&v)[COLS]) {
#pragma unroll
    for (int c = 0; c < COLS / 32; ++c) load32(at + 32 * c, reinterpret_cast<float (&)[32]>(v[32 * c]));
#pragma unroll
    for (int c = 0; c < COLS / 32; ++c) loaded(reinterpret_cast<float (&)[32]>(v[32 * c]));
}
template <int COLS>
__device__ __forceinline__ void store_cols(uint32_t at, const uint32_t (&w)[COLS / 2]) {
#pragma unroll
    for (int c = 0; c < COLS / 32; ++c) store16(at + 16 * c, w + 16 * c);
    stored();
}

struct GradArgs {
    AttnArgs g;
    uint64_t wait_ns;
    float scale2;                // scale log2 e
    int32_t vec;                 // rows of the outputs start on 16-byte boundaries
    int32_t parts;               // (keys) parts of a key head's query heads, each with its own sums
    float* part;                 // (keys) parts > 1: [part][dk, dv][k_rows][kv_heads dim]
    int32_t kv_items;            // CTAs of k_tc_grad that take keys, the first ones; the others take queries
};

// A CTA's rows done over in binary32 (iso_attn_simt.cuh), by 256 of its threads.
// Not inlined: nothing of it is held in registers before.
template <int DP>
__device__ __noinline__ void again_kv(const GradArgs& a, float* smem) {
    const AttnArgs& g = a.g;
    const int kv_heads = g.heads / g.group, part = blockIdx.x % a.parts, kh = blockIdx.x / a.parts % kv_heads;
    const int h0 = kh * g.group + g.group * part / a.parts, h1 = kh * g.group + g.group * (part + 1) / a.parts;
    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / a.parts / kv_heads, ROWS, true, t)) return;
    const long long width = (long long)kv_heads * g.head_dim;
    float* const o = a.part + (long long)(part * 2) * g.k_rows * width;
    for (const int last = t.first + min(ROWS, t.nk - t.first); t.first < last; t.first += SA_B) {
        if (a.parts > 1)
            simt_grad_kv<__nv_bfloat16, DP, float>(g, t, kh, h0, h1, o, width, o + g.k_rows * width, width, smem);
        else
            simt_grad_kv<__nv_bfloat16, DP, __nv_bfloat16>(g, t, kh, h0, h1, static_cast<__nv_bfloat16*>(g.dk), g.lddk,
                                                           static_cast<__nv_bfloat16*>(g.dv), g.lddv, smem);
        sa_sync();
    }
}
template <int DP>
__device__ __noinline__ void again_q(const GradArgs& a, float* smem) {
    const int index = (int)blockIdx.x - a.kv_items;
    AttnTile t;
    if (!attn_find_tile(a.g, index / a.g.heads, ROWS, false, t)) return;
    for (const int last = t.first + min(ROWS, t.nq - t.first); t.first < last; t.first += SA_B) {
        simt_grad_q<__nv_bfloat16, DP>(a.g, t, index % a.g.heads, smem);
        sa_sync();
    }
}

template <int DP>
__device__ __forceinline__ void grad_kv(const GradMaps& maps, const GradArgs& a, unsigned char* smem) {
    constexpr int TILE = GradTile<DP>::TILE;
    unsigned char *const sk = smem, *const sv = sk + TILE, *const sq = sv + TILE, *const sd = sq + KV_Q_STAGES * TILE;
    float* const lse_s = reinterpret_cast<float*>(sd + KV_DO_STAGES * TILE);
    float* const delta_s = lse_s + ROWS;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(delta_s + ROWS);
    const uint32_t bar = smem_u32(bars);
    const uint32_t k_full = bar, v_full = bar + 8, s_full = bar + 16, dp_full = bar + 24, p_ready = bar + 32,
                   ds_ready = bar + 40, lse_full = bar + 48, lse_empty = bar + 56, delta_full = bar + 64,
                   delta_empty = bar + 72, done = bar + 80, done2 = bar + 88, cleared = bar + 96 /* two */, rings = bar + 112;
    auto q_full = [&](int s) { return rings + 8u * s; };
    auto q_empty = [&](int s) { return rings + 8u * (KV_Q_STAGES + s); };
    auto do_full = [&](int s) { return rings + 8u * (2 * KV_Q_STAGES + s); };
    auto do_empty = [&](int s) { return rings + 8u * (2 * KV_Q_STAGES + KV_DO_STAGES + s); };
    constexpr int RINGS = 2 * (KV_Q_STAGES + KV_DO_STAGES);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(bars + 14 + RINGS);
    volatile int* const gave_up = reinterpret_cast<volatile int*>(slot + 1);
    volatile int* const again = gave_up + 1;           // a sum was not finite
    const AttnArgs& g = a.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kv_heads = g.heads / g.group;
    const int part = blockIdx.x % a.parts, kh = blockIdx.x / a.parts % kv_heads;

    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / a.parts / kv_heads, ROWS, true, t)) return;
    const int keys = min(ROWS, t.nk - t.first);
    int lo, hi, unused;
    attn_queries_of(g, t, t.first, lo, unused);
    attn_queries_of(g, t, t.first + keys - 1, unused, hi);
    const int tile0 = lo / ROWS, tiles = hi > lo ? (hi + ROWS - 1) / ROWS - tile0 : 0;
    const int h0 = kh * g.group + g.group * part / a.parts, h1 = kh * g.group + g.group * (part + 1) / a.parts;
    const int steps = (h1 - h0) * tiles;

    if (warp == GR_COMPUTE && lane == 0) {
        for (uint32_t b : {k_full, v_full, s_full, dp_full, lse_full, delta_full, done, done2}) mbar_init(b, 1);
        for (uint32_t b : {p_ready, ds_ready, lse_empty, delta_empty}) mbar_init(b, GR_COMPUTE);
        mbar_init(cleared, 1);
        mbar_init(cleared + 8, 1);
        for (int s = 0; s < KV_Q_STAGES; ++s) {
            mbar_init(q_full(s), 1);
            mbar_init(q_empty(s), 1);
        }
        for (int s = 0; s < KV_DO_STAGES; ++s) {
            mbar_init(do_full(s), 1);
            mbar_init(do_empty(s), 2);           // dP's products and dV's
        }
        *gave_up = *again = 0;
        mbar_fence_init();
        if (steps > 0) {                         // the first copies, while the CTA gets ready
            load_tile<DP>(smem_u32(sk), &maps.k, kh, t.k0 + t.first, k_full);
            load_tile<DP>(smem_u32(sq), &maps.q, h0, t.q0 + tile0 * ROWS, q_full(0));
            load_tile<DP>(smem_u32(sv), &maps.v, kh, t.k0 + t.first, v_full);
            load_tile<DP>(smem_u32(sd), &maps.dout, h0, t.q0 + tile0 * ROWS, do_full(0));
        }
    }
    if (warp == 0) alloc_all(smem_u32(slot));
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(slot);
    const uint32_t S = tmem, dP = tmem + 128, dV = tmem + 256, dK = tmem + 384;
    const Waits wait = {a.wait_ns, gave_up};

    if (warp == GR_COMPUTE) {
        // copies, of the second step on
        if (lane == 0 && steps > 0) {
            int nq = 1, nd = 1, h = h0, n = 0;
            for (int i = 1; i < steps; ++i) {
                if (++n == tiles) {
                    n = 0;
                    ++h;
                }
                const int row = t.q0 + (tile0 + n) * ROWS, qs = nq % KV_Q_STAGES, ds = nd % KV_DO_STAGES;
                if (!wait(q_empty(qs), (uint32_t)(nq / KV_Q_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sq) + qs * TILE, &maps.q, h, row, q_full(qs));
                ++nq;
                if (!wait(do_empty(ds), (uint32_t)(nd / KV_DO_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sd) + ds * TILE, &maps.dout, h, row, do_full(ds));
                ++nd;
            }
            // no copy is in flight when the CTA ends, after a give-up either
            wait.drain(k_full, 0);
            wait.drain(v_full, 0);
            for (int i = max(0, nq - KV_Q_STAGES); i < nq; ++i) wait.drain(q_full(i % KV_Q_STAGES), (uint32_t)(i / KV_Q_STAGES) & 1u);
            for (int i = max(0, nd - KV_DO_STAGES); i < nd; ++i) wait.drain(do_full(i % KV_DO_STAGES), (uint32_t)(i / KV_DO_STAGES) & 1u);
        }
    } else if (warp == GR_COMPUTE + 1) {
        // products of the weights: dV(i), then S^T(i + 1) over them.  (A whole warp waits
        // and clears, one lane issues.)
        Slot<KV_Q_STAGES> qn;                                                      // Q of the next scores
        Slot<KV_DO_STAGES> di;
        int tile = 0, tile_i = 0, tails = 0;                                       // its tile, step i's, last tiles so far
        const uint32_t k_s = smem_u32(sk), q_s = smem_u32(sq), d_s = smem_u32(sd);
        auto scores = [&] {                                                        // S^T = K Q^T
            if (!wait.warp(q_full(qn.at), qn.parity)) return false;
            if (tile == tiles - 1) clear_rows<DP>(sq + qn.at * TILE, t.nq - (tile0 + tile) * ROWS);
            after_sync();
            if (elected()) {
                product_along<DP>(S, k_s, q_s + (uint32_t)qn.at * TILE);
                commit(s_full);
            }
            __syncwarp();
            qn.next();
            if (++tile == tiles) tile = 0;
            return true;
        };
        bool ok = steps > 0 && wait.warp(k_full, 0) && scores();
        for (int i = 0; ok && i < steps; ++i) {
            // dO is there, and where it had to be cleared, cleared (by the other warp)
            if (!(ok = wait.warp(do_full(di.at), di.parity))) break;
            if (++tile_i == tiles) {
                tile_i = 0;
                if (!(ok = wait.warp(cleared + 8u * (tails & 1), (uint32_t)(tails >> 1) & 1u))) break;
                ++tails;
            }
            if (!(ok = wait.warp(p_ready, (uint32_t)i & 1u))) break;
            after_sync();
            if (elected()) {
                product_rows<DP, GR_COLS>(dV, S, d_s + (uint32_t)di.at * TILE, i > 0);
                commit(do_empty(di.at));
            }
            __syncwarp();
            di.next();
            if (i + 1 < steps) ok = scores();
        }
        // no product runs on when the tensor memory is freed, after a give-up either
        if (steps > 0 && elected()) {
            commit(done);
            wait.drain(done, 0);
        }
    } else if (warp == GR_COMPUTE + 2) {
        // products of the scores' gradients: dK(i), then dP^T(i + 1) over them
        Slot<KV_DO_STAGES> dn;
        Slot<KV_Q_STAGES> qi;
        int tile = 0, tails = 0;
        const uint32_t v_s = smem_u32(sv), q_s = smem_u32(sq), d_s = smem_u32(sd);
        auto values = [&] {                                                        // dP^T = V dO^T
            if (!wait.warp(do_full(dn.at), dn.parity)) return false;
            if (tile == tiles - 1) {
                clear_rows<DP>(sd + dn.at * TILE, t.nq - (tile0 + tile) * ROWS);
                arrive_warp(cleared + 8u * (tails++ & 1));
            }
            after_sync();
            if (elected()) {
                product_along<DP>(dP, v_s, d_s + (uint32_t)dn.at * TILE);
                commit(dp_full);
                commit(do_empty(dn.at));
            }
            __syncwarp();
            dn.next();
            if (++tile == tiles) tile = 0;
            return true;
        };
        bool ok = steps > 0 && wait.warp(v_full, 0) && values();
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = wait.warp(ds_ready, (uint32_t)i & 1u))) break;
            after_sync();
            if (elected()) {
                product_rows<DP, GR_COLS>(dK, dP, q_s + (uint32_t)qi.at * TILE, i > 0);
                commit(q_empty(qi.at));
            }
            __syncwarp();
            qi.next();
            if (i + 1 < steps) ok = values();
        }
        if (steps > 0 && elected()) {
            commit(done2);
            wait.drain(done2, 0);
        }
    } else if (warp == GR_COMPUTE + 3) {
        // -lse log2 e and -delta of a step's queries: four a lane.  A query behind the
        // sequence's end has an infinite lse, so that its weights are 0.
        int i = 0;
        bool ok = true;
        for (int h = h0; ok && h < h1; ++h)
            for (int n = 0; n < tiles; ++n, ++i) {
                const int first = (tile0 + n) * ROWS + lane;
                const long long at = (long long)h * g.q_rows + t.q0 + first;
                float l[4], d[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = first + 32 * j < t.nq;
                    l[j] = in ? -g.lse[at + 32 * j] * LOG2E : -INFINITY;
                    d[j] = in ? -g.delta[at + 32 * j] : 0.0f;
                }
                if (!(ok = wait.warp(lse_empty, (uint32_t)(i + 1) & 1u))) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) lse_s[lane + 32 * j] = l[j];
                arrive_warp(lse_full);
                if (!(ok = wait.warp(delta_empty, (uint32_t)(i + 1) & 1u))) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) delta_s[lane + 32 * j] = d[j];
                arrive_warp(delta_full);
            }
    } else {
        // A thread has four rows of a quarter of the columns (as load_rows16 gives
        // them), so that it needs lse and delta of 16 columns, eight bytes a load: with a row
        // a thread it is 64 of each, in loads that are broadcasts and cost shared memory
        // what as many different words would (a step's weights 1154 -> 753 clocks, its dS
        // 835 -> 512).
        const int group = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t at = ((uint32_t)(warp & 3) * 32) << 16, low = 16u << 16;
        const uint32_t s_at = S + at + group * GR_COLS, d_at = dP + at + group * GR_COLS;
        int from[4], to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            attn_queries_of(g, t, t.first + min((warp & 3) * 32 + 8 * j + (lane >> 2), keys - 1), from[j], to[j]);
        const uint64_t c = pair_of(a.scale2, a.scale2);
        const uint64_t* const neg_lse = reinterpret_cast<const uint64_t*>(lse_s + group * GR_COLS) + (lane & 3);
        const uint64_t* const neg_delta = reinterpret_cast<const uint64_t*>(delta_s + group * GR_COLS) + (lane & 3);
        bool ok = true;
        const int column0 = tile0 * ROWS + group * GR_COLS;
        for (int i = 0, n = 0; i < steps; ++i, n = n + 1 == tiles ? 0 : n + 1) {
            const uint32_t ph = (uint32_t)i & 1u;
            const int q0 = column0 + n * ROWS;
            bool whole = true;                                    // every column of every row is seen
#pragma unroll
            for (int j = 0; j < 4; ++j) whole = whole && from[j] <= q0 && to[j] >= q0 + GR_COLS;
            const bool masked = !__all_sync(0xFFFFFFFFu, whole);
            // of this thread's rows 8 j + lane / 4 and its columns: seen(j, column)
            auto seen = [&](int j, int col) { return q0 + col >= from[j] && q0 + col < to[j]; };
            uint64_t p[2][16];
            float v[2][32];
            uint32_t w[2][16];
            if (!(ok = wait.warp(lse_full, ph) && wait.warp(s_full, ph))) break;
            after_sync();
            load_rows16(s_at, v[0]);
            load_rows16(s_at + low, v[1]);
            loaded(v[0]);
            loaded(v[1]);
            auto weights = [&](auto mask) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint64_t l = neg_lse[4 * k];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x, y;
                        parts_of(fma2(pair_of(v[j / 2][4 * k + 2 * (j & 1)], v[j / 2][4 * k + 2 * (j & 1) + 1]), c, l), x, y);
                        x = ex2(x);
                        y = ex2(y);
                        if (decltype(mask)::value && !seen(j, 8 * k + 2 * (lane & 3))) x = 0.0f;
                        if (decltype(mask)::value && !seen(j, 8 * k + 2 * (lane & 3) + 1)) y = 0.0f;
                        p[j / 2][2 * k + (j & 1)] = pair_of(x, y);
                        w[j / 2][2 * k + (j & 1)] = f32_to_bf16x2(x, y);
                    }
                }
            };
            if (masked) weights(std::true_type{});
            else weights(std::false_type{});
            store_rows16(s_at, w[0]);
            store_rows16(s_at + low, w[1]);
            stored();
            before_sync();
            arrive_warp(p_ready);
            if (lane == 0) mbar_arrive(lse_empty);
            if (!(ok = wait.warp(delta_full, ph) && wait.warp(dp_full, ph))) break;
            after_sync();
            load_rows16(d_at, v[0]);
            load_rows16(d_at + low, v[1]);
            loaded(v[0]);
            loaded(v[1]);
            auto score_grads = [&](auto mask) {                   // (what is not seen is 0 whatever dP is there)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint64_t d = neg_delta[4 * k];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x, y;
                        parts_of(mul2(add2(pair_of(v[j / 2][4 * k + 2 * (j & 1)], v[j / 2][4 * k + 2 * (j & 1) + 1]), d),
                                      p[j / 2][2 * k + (j & 1)]), x, y);
                        if (decltype(mask)::value && !seen(j, 8 * k + 2 * (lane & 3))) x = 0.0f;
                        if (decltype(mask)::value && !seen(j, 8 * k + 2 * (lane & 3) + 1)) y = 0.0f;
                        w[j / 2][2 * k + (j & 1)] = f32_to_bf16x2(x, y);
                    }
                }
            };
            if (masked) score_grads(std::true_type{});
            else score_grads(std::false_type{});
            store_rows16(d_at, w[0]);
            store_rows16(d_at + low, w[1]);
            stored();
            before_sync();
            arrive_warp(ds_ready);
            if (lane == 0) mbar_arrive(delta_empty);
        }
        // dV by the first half of the warps, dK by the second: a row a thread
        const int half = group;
        if (steps > 0) ok = ok && wait.warp(half ? done2 : done, 0);
        after_sync();
        const bool nan = !ok || (steps > 0 && *gave_up), none = steps == 0;
        const uint32_t acc = (half ? dK : dV) + at;
        const float by = half ? g.scale : 1.0f;
        const long long row = (long long)t.k0 + t.first + r;
        if (a.parts > 1) {
            const long long width = (long long)kv_heads * g.head_dim;
            float* o = a.part + ((long long)(part * 2 + (half ? 0 : 1)) * g.k_rows + row) * width + (long long)kh * g.head_dim;
            if (!write_row<float, DP>(acc, o, r < keys, g.head_dim, true, by, nan, none)) *again = 1;
        } else {
            __nv_bfloat16* o = static_cast<__nv_bfloat16*>(half ? g.dk : g.dv) + row * (half ? g.lddk : g.lddv) + (long long)kh * g.head_dim;
            if (!write_row<__nv_bfloat16, DP>(acc, o, r < keys, g.head_dim, a.vec, by, nan, none)) *again = 1;
        }
        before_sync();
    }
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        after_sync();
        free_all(tmem);
    }
    if (*again && !*gave_up && warp < SA_TPB / 32) again_kv<DP>(a, reinterpret_cast<float*>(smem));
}

template <int DP>
__device__ __forceinline__ void grad_q(const GradMaps& maps, const GradArgs& a, unsigned char* smem) {
    constexpr int TILE = GradTile<DP>::TILE;
    const int index = (int)blockIdx.x - a.kv_items;
    unsigned char *const sq = smem, *const sd = sq + TILE, *const sk = sd + TILE, *const sv = sk + Q_K_STAGES * TILE;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(sv + Q_V_STAGES * TILE);
    const uint32_t bar = smem_u32(bars);
    const uint32_t q_full = bar, do_full = bar + 8, s_full = bar + 16 /* two */, dp_full = bar + 32, ds_ready = bar + 40 /* two */,
                   done = bar + 56, done2 = bar + 64, rings = bar + 72;
    auto k_full = [&](int s) { return rings + 8u * s; };
    auto k_empty = [&](int s) { return rings + 8u * (Q_K_STAGES + s); };
    auto v_full = [&](int s) { return rings + 8u * (2 * Q_K_STAGES + s); };
    auto v_empty = [&](int s) { return rings + 8u * (2 * Q_K_STAGES + Q_V_STAGES + s); };
    constexpr int RINGS = 2 * (Q_K_STAGES + Q_V_STAGES);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(bars + 9 + RINGS);
    volatile int* const gave_up = reinterpret_cast<volatile int*>(slot + 1);
    volatile int* const again = gave_up + 1;           // a sum was not finite
    const AttnArgs& g = a.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = index % g.heads, kh = h / g.group;

    AttnTile t;
    if (!attn_find_tile(g, index / g.heads, ROWS, false, t)) return;
    const int rows = min(ROWS, t.nq - t.first);
    int lo, hi, unused;
    attn_keys_of(g, t, t.first, lo, unused);
    attn_keys_of(g, t, t.first + rows - 1, unused, hi);
    const int tile0 = lo / ROWS, steps = hi > lo ? (hi + ROWS - 1) / ROWS - tile0 : 0;

    if (warp == GR_COMPUTE && lane == 0) {
        for (uint32_t b : {q_full, do_full, s_full, s_full + 8, dp_full, done, done2}) mbar_init(b, 1);
        mbar_init(ds_ready, GR_COMPUTE);
        mbar_init(ds_ready + 8, GR_COMPUTE);
        for (int s = 0; s < RINGS; ++s) mbar_init(rings + 8u * s, 1);
        *gave_up = *again = 0;
        mbar_fence_init();
        if (steps > 0) {                         // the first copies, while the CTA gets ready
            load_tile<DP>(smem_u32(sq), &maps.q, h, t.q0 + t.first, q_full);
            load_tile<DP>(smem_u32(sk), &maps.k, kh, t.k0 + tile0 * ROWS, k_full(0));
            load_tile<DP>(smem_u32(sd), &maps.dout, h, t.q0 + t.first, do_full);
            load_tile<DP>(smem_u32(sv), &maps.v, kh, t.k0 + tile0 * ROWS, v_full(0));
        }
    }
    if (warp == 0) alloc_all(smem_u32(slot));
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(slot);
    const uint32_t S = tmem, dP = tmem + 256, dQ = tmem + 384;       // S: two buffers of 128 columns
    const Waits wait = {a.wait_ns, gave_up};

    if (warp == GR_COMPUTE) {
        if (lane == 0 && steps > 0) {
            int nk = 1, nv = 1;
            for (int n = 1; n < steps; ++n) {
                const int row = t.k0 + (tile0 + n) * ROWS, ks = nk % Q_K_STAGES, vs = nv % Q_V_STAGES;
                if (!wait(k_empty(ks), (uint32_t)(nk / Q_K_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sk) + ks * TILE, &maps.k, kh, row, k_full(ks));
                ++nk;
                if (!wait(v_empty(vs), (uint32_t)(nv / Q_V_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sv) + vs * TILE, &maps.v, kh, row, v_full(vs));
                ++nv;
            }
            wait.drain(q_full, 0);
            wait.drain(do_full, 0);
            for (int i = max(0, nk - Q_K_STAGES); i < nk; ++i) wait.drain(k_full(i % Q_K_STAGES), (uint32_t)(i / Q_K_STAGES) & 1u);
            for (int i = max(0, nv - Q_V_STAGES); i < nv; ++i) wait.drain(v_full(i % Q_V_STAGES), (uint32_t)(i / Q_V_STAGES) & 1u);
        }
    } else if (warp == GR_COMPUTE + 1) {
        // dQ(i), then S(i + 2) over its weights.  (A whole warp waits and clears, one
        // lane issues.)
        Slot<Q_K_STAGES> kn, ki;
        const uint32_t q_s = smem_u32(sq), k_s = smem_u32(sk);
        int next = 0;                                                              // the next scores
        auto scores = [&] {                                                        // S = Q K^T
            if (!wait.warp(k_full(kn.at), kn.parity)) return false;
            if (next == steps - 1) clear_rows<DP>(sk + kn.at * TILE, t.nk - (tile0 + next) * ROWS);
            after_sync();
            if (elected()) {
                product_along<DP>(S + (next & 1) * 128, q_s, k_s + (uint32_t)kn.at * TILE);
                commit(s_full + 8u * (next & 1));
            }
            __syncwarp();
            kn.next();
            ++next;
            return true;
        };
        bool ok = steps > 0 && wait.warp(q_full, 0) && scores() && (steps < 2 || scores());
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = wait.warp(ds_ready + 8u * (i & 1), (uint32_t)(i >> 1) & 1u))) break;
            after_sync();
            if (elected()) {
                product_rows<DP, GR_COLS>(dQ, S + (i & 1) * 128, k_s + (uint32_t)ki.at * TILE, i > 0);
                commit(k_empty(ki.at));
            }
            __syncwarp();
            ki.next();
            if (i + 2 < steps) ok = scores();
        }
        // no product runs on when the tensor memory is freed, after a give-up either
        if (steps > 0 && elected()) {
            commit(done);
            wait.drain(done, 0);
        }
    } else if (warp == GR_COMPUTE + 2) {
        // dP(i + 1) once dP(i) has been read
        Slot<Q_V_STAGES> vn;
        const uint32_t d_s = smem_u32(sd), v_s = smem_u32(sv);
        bool ok = steps > 0 && wait.warp(do_full, 0);
        for (int i = 0; ok && i < steps; ++i) {
            if (i > 0 && !(ok = wait.warp(ds_ready + 8u * ((i - 1) & 1), (uint32_t)((i - 1) >> 1) & 1u))) break;
            if (!(ok = wait.warp(v_full(vn.at), vn.parity))) break;
            after_sync();
            if (elected()) {
                product_along<DP>(dP, d_s, v_s + (uint32_t)vn.at * TILE);          // dP = dO V^T
                commit(dp_full);
                commit(v_empty(vn.at));
            }
            __syncwarp();
            vn.next();
        }
        if (steps > 0 && elected()) {
            commit(done2);
            wait.drain(done2, 0);
        }
    } else if (warp < GR_COMPUTE) {
        const int group = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t at = ((uint32_t)(warp & 3) * 32) << 16, d_at = dP + at + group * GR_COLS;
        int from, to;
        attn_keys_of(g, t, t.first + min(r, rows - 1), from, to);
        const long long stat = (long long)h * g.q_rows + t.q0 + t.first + min(r, rows - 1);
        const float neg_lse = -g.lse[stat] * LOG2E, neg_delta = -g.delta[stat];
        const uint64_t c = pair_of(a.scale2, a.scale2), ll = pair_of(neg_lse, neg_lse), dd = pair_of(neg_delta, neg_delta);
        bool ok = true;
        for (int i = 0; i < steps; ++i) {
            const uint32_t s_at = S + (i & 1) * 128 + at + group * GR_COLS;
            const int k0 = (tile0 + i) * ROWS + group * GR_COLS;
            const int f = from - k0, e = to - k0;
            const bool masked = !__all_sync(0xFFFFFFFFu, f <= 0 && e >= GR_COLS);
            uint64_t p[GR_COLS / 2];
            float v[GR_COLS];
            uint32_t w[GR_COLS / 2];
            if (!(ok = wait.warp(s_full + 8u * (i & 1), (uint32_t)(i >> 1) & 1u))) break;
            after_sync();
            load_cols<GR_COLS>(s_at, v);
            if (masked) weights<true, GR_COLS>(v, p, c, f, e, [&](int) { return ll; });
            else weights<false, GR_COLS>(v, p, c, f, e, [&](int) { return ll; });
            if (!(ok = wait.warp(dp_full, (uint32_t)i & 1u))) break;
            after_sync();
            load_cols<GR_COLS>(d_at, v);
            if (masked) score_grads<true, GR_COLS>(v, p, w, f, e, [&](int) { return dd; });
            else score_grads<false, GR_COLS>(v, p, w, f, e, [&](int) { return dd; });
            store_cols<GR_COLS>(s_at, w);
            before_sync();
            arrive_warp(ds_ready + 8u * (i & 1));
        }
        if (steps > 0 && ok) wait.warp(done, 0);
        after_sync();
        // dQ: a row a thread, some columns of it each group; both groups know whether one of
        // them gave up, so that a row is whole or NaN
        sa_sync();
        constexpr int WIDE = DP * 4 / GR_COMPUTE;
        const bool nan = *gave_up, none = steps == 0;
        const int from_col = group * WIDE;
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(g.dq) + ((long long)t.q0 + t.first + r) * g.lddq + (long long)h * g.head_dim + from_col;
        if (!write_row<__nv_bfloat16, WIDE>(dQ + at + from_col, o, r < rows, g.head_dim - from_col, a.vec, g.scale, nan, none))
            *again = 1;
        before_sync();
    }
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        after_sync();
        free_all(tmem);
    }
    if (*again && !*gave_up && warp < SA_TPB / 32) again_q<DP>(a, reinterpret_cast<float*>(smem));
}

// One launch for both, keys first: the CTAs of queries fill the SMs that the last
// ones of keys leave (8192 tokens, 28 heads over 4 of 128, three parts, with the first
// copies before the CTA is ready: 1138 -> 1062 us; 13 packed sequences of 12 heads over
// 2: 180 -> 153 us).
template <int DP>
__global__ void __launch_bounds__(GR_THREADS, 1) k_tc_grad(const __grid_constant__ GradMaps maps, const __grid_constant__ GradArgs a) {
    extern __shared__ unsigned char gr_smem_raw[];
    if ((int)blockIdx.x < a.kv_items) grad_kv<DP>(maps, a, align1024(gr_smem_raw));
    else grad_q<DP>(maps, a, align1024(gr_smem_raw));
}

// dk and dv: the parts' sums in order.  Eight columns a thread.
template <bool VEC>
__global__ void __launch_bounds__(256) k_grad_join(const __grid_constant__ GradArgs a) {
    const AttnArgs& g = a.g;
    const int width = g.heads / g.group * g.head_dim, segs = width / 8;
    int first = 0, last = g.k_rows;
    if (g.n_seqs) {
        first = min(max(g.k_ends[0], 0), g.k_rows);
        last = min(max(g.k_ends[g.n_seqs], 0), g.k_rows);
    }
    const long long n = (long long)max(last - first, 0) * segs;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < 2 * n; i += (long long)gridDim.x * blockDim.x) {
        const bool v = i >= n;
        const long long at = v ? i - n : i, row = first + at / segs;
        const int c = (int)(at % segs) * 8;
        float s[8] = {};
        for (int p = 0; p < a.parts; ++p) {
            float x[8];
            load8<true>(a.part + ((long long)(p * 2 + v) * g.k_rows + row) * width, c, width, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += x[j];
        }
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(v ? g.dv : g.dk) + row * (v ? g.lddv : g.lddk);
        store8<VEC>(o, c, width, s);
    }
}

template <int DP>
int launch_grad(const GradMaps& m, GradArgs a, cudaStream_t s) {
    constexpr int SMEM = std::max(GradTile<DP>::KV_SMEM, GradTile<DP>::Q_SMEM);
    const AttnArgs& g = a.g;
    const long long kv = attn_tiles(g.k_rows, g.n_seqs, ROWS) * (g.heads / g.group) * a.parts;
    const long long q = attn_tiles(g.q_rows, g.n_seqs, ROWS) * g.heads;
    if (kv + q > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    a.kv_items = (int)kv;
    static std::atomic<uint64_t> done{0};
    ISO_TRY(allow_smem(k_tc_grad<DP>, SMEM, done));
    TRAIN_LAUNCH((k_tc_grad<DP><<<(unsigned)(kv + q), GR_THREADS, SMEM, s>>>(m, a)));
    return ISO_OK;
}

}  // namespace

// Parts by the estimated time: the average SM's, with a tenth of the longest CTA for
// the end, or that CTA's where it is longer; and the parts' sums written and read
// again.  From the sizes alone, a packed sequence taken as of average length and the
// longest as twice that.  Measured (heads of 128, causal), one, two and three parts:
// 8192 tokens, 28 heads over 4: 1029 / 1063 / 1083 us; 12 over 2: 540 / 464 / 474;
// 2048 tokens, 12 over 2: 148 / 87 / 67 (six: 65); 13 sequences of 8192 tokens in
// all, 12 over 2: 127 / 141 / 152; 512 tokens, 28 over 4: 57 / 44 / 38 (seven: 35).
AttnGradPlan attn_grad_plan(long long q_rows, long long k_rows, const iso_attn_cfg& c) {
    const int group = c.heads / c.kv_heads;
    const long long seqs = std::max(1, c.n_seqs), sms = train_sms();
    const double k_tiles = (double)((k_rows + ROWS - 1) / ROWS), q_tiles = (double)((q_rows + ROWS - 1) / ROWS);
    const double of_seq = std::max(1.0, (double)q_rows / seqs / ROWS);                  // query tiles of a sequence
    const double longest = seqs > 1 ? 2.0 * of_seq : of_seq;
    const double total = k_tiles * c.heads * (c.causal ? 0.5 * (of_seq + 1.0) : of_seq);
    AttnGradPlan p{1, 0};
    double best = 0.0;
    for (int parts = 1; parts <= group; ++parts) {
        const double item = longest * ((group + parts - 1) / parts), items = k_tiles * c.kv_heads * parts + q_tiles * c.heads;
        const double average = (total * (1.0 + GR_Q_STEP) + GR_ITEM_STEPS * items) / sms;
        const double join = parts == 1 ? 0.0 : GR_JOIN_STEPS + (double)k_rows * c.kv_heads * c.head_dim * 16.0 * parts / GR_STEP_BYTES;
        const double cost = std::max(average + 0.1 * item, item + GR_ITEM_STEPS) + join;
        if (parts == 1 || cost < best) {
            best = cost;
            p.parts = parts;
        }
    }
    p.bytes = p.parts > 1 ? (size_t)p.parts * 2 * k_rows * c.kv_heads * c.head_dim * 4 : 0;
    return p;
}

int attn_grad_tc(const AttnArgs& g, const AttnGradPlan& p, float* part, cudaStream_t s) {
    GradMaps m;
    ISO_TRY(tc::head_map(&m.q, g.q, g.q_rows, g.heads, g.head_dim, g.ldq));
    ISO_TRY(tc::head_map(&m.k, g.k, g.k_rows, g.heads / g.group, g.head_dim, g.ldk));
    ISO_TRY(tc::head_map(&m.v, g.v, g.k_rows, g.heads / g.group, g.head_dim, g.ldv));
    ISO_TRY(tc::head_map(&m.dout, g.dout, g.q_rows, g.heads, g.head_dim, g.lddo));
    auto aligned = [](const void* p, long long ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0; };
    GradArgs a{};
    a.g = g;
    a.wait_ns = attn_wait_ns();
    a.scale2 = g.scale * LOG2E;
    a.vec = aligned(g.dq, g.lddq) && aligned(g.dk, g.lddk) && aligned(g.dv, g.lddv);
    a.parts = p.parts;
    a.part = part;
    ISO_TRY(g.head_dim <= 64 ? launch_grad<64>(m, a, s) : launch_grad<128>(m, a, s));
    if (p.parts == 1 || g.k_rows == 0) return ISO_OK;
    const long long n = 2LL * g.k_rows * (g.heads / g.group) * g.head_dim / 8;
    const unsigned grid = (unsigned)std::min<long long>((n + 255) / 256, 1 << 20);
    TRAIN_LAUNCH((a.vec ? k_grad_join<true><<<grid, 256, 0, s>>>(a) : k_grad_join<false><<<grid, 256, 0, s>>>(a)));
    return ISO_OK;
}

}  // namespace iso
