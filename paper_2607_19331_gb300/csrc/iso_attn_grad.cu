// iso_attn_grad.cu -- attention's gradients on the fifth-generation tensor cores
// (bfloat16, head dimensions up to 128).
//
// The weights are formed again from lse, and both kernels own what they write, so
// there are no atomics and no binary32 gradients in memory; that takes seven products of
// 128 x 128 x dim a pair of tiles instead of five.
//   k_tc_grad_kv   128 keys: over the query tiles (and query heads) that see them
//                    S^T = K Q^T       P^T = exp2(c S^T - lse2)      dV += P^T dO
//                    dP^T = V dO^T     dS^T = P^T (dP^T - delta)     dK += dS^T Q
//                  Keys are rows, so that P^T and dS^T, rounded to bf16, go back
//                  to tensor memory over the scores they came from and are the A
//                  operands of the second products as they are; Q and dO serve
//                  both as rows to contract along and as rows to contract over.
//                  The products are issued as
//                    dV(i) S(i+1) | dK(i) dP(i+1) | dV(i+1) ...
//                  so that while the warps form P(i+1) from S(i+1) the pair dK(i),
//                  dP(i+1) runs, and while they form dS(i+1), the pair dV(i+1),
//                  S(i+2): one buffer each for scores and dP keeps both busy.
//   k_tc_grad_q    128 queries: over the key tiles that they see
//                    S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//                  with two buffers of scores; dS lies over its scores.
// Tensor memory is full in both (4 x 128 columns).
// Eight warps compute, four on each half of a tile's columns; one warp copies,
// one issues products; in k_tc_grad_kv one more brings lse and delta, which are
// per column there.
#include "iso_attn.cuh"
#include "iso_attn_simt.cuh"
#include "iso_attn_tc.cuh"
#include "iso_tc.cuh"

#include <algorithm>
#include <atomic>

namespace iso {
namespace {

using namespace tc;

constexpr int GR_COMPUTE = 8;
constexpr int GR_THREADS = (GR_COMPUTE + 3) * 32;
constexpr int KV_Q_STAGES = 3, KV_DO_STAGES = 2, Q_K_STAGES = 3, Q_V_STAGES = 2;

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

// The 64 weights of this thread's row and half: p = exp2(c s - lse2), 0 outside
// [from, to) where the tile is masked
template <bool MASKED>
__device__ __forceinline__ float weight(float s, float c, float lse2, int at, int from, int to) {
    const float p = ex2(fmaf(s, c, -lse2));
    return !MASKED || (at >= from && at < to) ? p : 0.0f;
}

struct GradArgs {
    AttnArgs g;
    uint64_t wait_ns;
    float scale2;                // scale log2 e
    int32_t vec;                 // rows of the outputs start on 16-byte boundaries
    int32_t parts;               // (keys) parts of a key head's query heads, each with its own sums
    float* part;                 // (keys) parts > 1: [part][dk, dv][k_rows][kv_heads dim]
};

template <int DP>
__global__ void __launch_bounds__(GR_THREADS, 1)
k_tc_grad_kv(const __grid_constant__ GradMaps maps, const __grid_constant__ GradArgs a) {
    constexpr int TILE = GradTile<DP>::TILE;
    extern __shared__ unsigned char gr_smem_raw[];
    unsigned char* const smem = align1024(gr_smem_raw);
    unsigned char *const sk = smem, *const sv = sk + TILE, *const sq = sv + TILE, *const sd = sq + KV_Q_STAGES * TILE;
    float* const lse_s = reinterpret_cast<float*>(sd + KV_DO_STAGES * TILE);
    float* const delta_s = lse_s + ROWS;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(delta_s + ROWS);
    const uint32_t bar = smem_u32(bars);
    const uint32_t k_full = bar, v_full = bar + 8, s_full = bar + 16, dp_full = bar + 24, p_ready = bar + 32,
                   ds_ready = bar + 40, lse_full = bar + 48, lse_empty = bar + 56, delta_full = bar + 64,
                   delta_empty = bar + 72, done = bar + 80, rings = bar + 88;
    auto q_full = [&](int s) { return rings + 8u * s; };
    auto q_empty = [&](int s) { return rings + 8u * (KV_Q_STAGES + s); };
    auto do_full = [&](int s) { return rings + 8u * (2 * KV_Q_STAGES + s); };
    auto do_empty = [&](int s) { return rings + 8u * (2 * KV_Q_STAGES + KV_DO_STAGES + s); };
    constexpr int RINGS = 2 * (KV_Q_STAGES + KV_DO_STAGES);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(bars + 11 + RINGS);
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

    if (threadIdx.x == 0) {
        for (uint32_t b : {k_full, v_full, s_full, dp_full, lse_full, delta_full, done}) mbar_init(b, 1);
        for (uint32_t b : {p_ready, ds_ready, lse_empty, delta_empty}) mbar_init(b, GR_COMPUTE);
        for (int s = 0; s < RINGS; ++s) mbar_init(rings + 8u * s, 1);
        *gave_up = *again = 0;
        mbar_fence_init();
    }
    if (warp == 0) alloc_all(smem_u32(slot));
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(slot);
    const uint32_t S = tmem, dP = tmem + 128, dV = tmem + 256, dK = tmem + 384;
    const Waits wait = {a.wait_ns, gave_up};

    if (warp == GR_COMPUTE) {
        // copies
        if (lane == 0 && steps > 0) {
            load_tile<DP>(smem_u32(sk), &maps.k, kh, t.k0 + t.first, k_full);
            int nq = 0, nd = 0;
            bool ok = true;
            for (int h = h0; ok && h < h1; ++h)
                for (int n = 0; n < tiles; ++n) {
                    const int row = t.q0 + (tile0 + n) * ROWS, qs = nq % KV_Q_STAGES, ds = nd % KV_DO_STAGES;
                    if (!(ok = wait(q_empty(qs), (uint32_t)(nq / KV_Q_STAGES + 1) & 1u))) break;
                    load_tile<DP>(smem_u32(sq) + qs * TILE, &maps.q, h, row, q_full(qs));
                    if (nq++ == 0) load_tile<DP>(smem_u32(sv), &maps.v, kh, t.k0 + t.first, v_full);
                    if (!(ok = wait(do_empty(ds), (uint32_t)(nd / KV_DO_STAGES + 1) & 1u))) break;
                    load_tile<DP>(smem_u32(sd) + ds * TILE, &maps.dout, h, row, do_full(ds));
                    ++nd;
                }
            // no copy is in flight when the CTA ends, after a give-up either
            wait.drain(k_full, 0);
            if (nq) wait.drain(v_full, 0);
            for (int i = max(0, nq - KV_Q_STAGES); i < nq; ++i) wait.drain(q_full(i % KV_Q_STAGES), (uint32_t)(i / KV_Q_STAGES) & 1u);
            for (int i = max(0, nd - KV_DO_STAGES); i < nd; ++i) wait.drain(do_full(i % KV_DO_STAGES), (uint32_t)(i / KV_DO_STAGES) & 1u);
        }
    } else if (warp == GR_COMPUTE + 1) {
        // products (the whole warp waits and clears, one lane issues)
        auto q_at = [&](int i) { return smem_u32(sq) + (uint32_t)(i % KV_Q_STAGES) * TILE; };
        auto do_at = [&](int i) { return smem_u32(sd) + (uint32_t)(i % KV_DO_STAGES) * TILE; };
        auto valid = [&](int i) { return t.nq - (tile0 + i % tiles) * ROWS; };     // rows of step i's query tile
        auto scores = [&](int i) {                                                 // S^T = K Q^T
            const int s = i % KV_Q_STAGES;
            if (!wait.warp(q_full(s), (uint32_t)(i / KV_Q_STAGES) & 1u)) return false;
            clear_rows<DP>(sq + s * TILE, valid(i));
            after_sync();
            if (lane == 0) {
                product_along<DP>(S, smem_u32(sk), q_at(i));
                commit(s_full);
            }
            __syncwarp();
            return true;
        };
        auto values = [&](int i) {                                                 // dP^T = V dO^T
            const int s = i % KV_DO_STAGES;
            if (!wait.warp(do_full(s), (uint32_t)(i / KV_DO_STAGES) & 1u)) return false;
            clear_rows<DP>(sd + s * TILE, valid(i));
            after_sync();
            if (lane == 0) {
                product_along<DP>(dP, smem_u32(sv), do_at(i));
                commit(dp_full);
            }
            __syncwarp();
            return true;
        };
        bool ok = steps > 0 && wait.warp(k_full, 0) && scores(0) && wait.warp(v_full, 0) && values(0);
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = wait.warp(p_ready, (uint32_t)i & 1u))) break;
            after_sync();
            if (lane == 0) {
                product_rows<DP>(dV, S, S + 64, do_at(i), i > 0);
                commit(do_empty(i % KV_DO_STAGES));
            }
            __syncwarp();
            if (i + 1 < steps && !(ok = scores(i + 1))) break;
            if (!(ok = wait.warp(ds_ready, (uint32_t)i & 1u))) break;
            after_sync();
            if (lane == 0) {
                product_rows<DP>(dK, dP, dP + 64, q_at(i), i > 0);
                commit(q_empty(i % KV_Q_STAGES));
            }
            __syncwarp();
            if (i + 1 < steps && !(ok = values(i + 1))) break;
        }
        // no product runs on when the tensor memory is freed, after a give-up either
        if (lane == 0 && steps > 0) {
            commit(done);
            wait.drain(done, 0);
        }
    } else if (warp == GR_COMPUTE + 2) {
        // lse and delta of a step's queries: four a lane.  A query behind the
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
                    l[j] = in ? g.lse[at + 32 * j] * LOG2E : INFINITY;
                    d[j] = in ? g.delta[at + 32 * j] : 0.0f;
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
        const int half = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t at = ((uint32_t)(warp & 3) * 32) << 16, s_at = S + at + half * 64, d_at = dP + at + half * 64;
        int from, to;
        attn_queries_of(g, t, t.first + min(r, keys - 1), from, to);
        bool ok = true;
        for (int i = 0; i < steps; ++i) {
            const uint32_t ph = (uint32_t)i & 1u;
            const int q0 = (tile0 + i % tiles) * ROWS + half * 64;
            const int f = from - q0, e = to - q0;                 // this thread's columns that are seen
            const bool masked = !__all_sync(0xFFFFFFFFu, f <= 0 && e >= 64);
            float p[64];
            if (!(ok = wait.warp(lse_full, ph) && wait.warp(s_full, ph))) break;
            after_sync();
            {
                float v[2][32];
                load32(s_at, v[0]);
                loaded(v[0]);
                load32(s_at + 32, v[1]);
                auto form = [&](auto m, int c) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(lse_s + half * 64 + c * 32 + j);
                        p[c * 32 + j] = weight<decltype(m)::value>(v[c][j], a.scale2, l.x, c * 32 + j, f, e);
                        p[c * 32 + j + 1] = weight<decltype(m)::value>(v[c][j + 1], a.scale2, l.y, c * 32 + j + 1, f, e);
                        p[c * 32 + j + 2] = weight<decltype(m)::value>(v[c][j + 2], a.scale2, l.z, c * 32 + j + 2, f, e);
                        p[c * 32 + j + 3] = weight<decltype(m)::value>(v[c][j + 3], a.scale2, l.w, c * 32 + j + 3, f, e);
                    }
                };
                uint32_t w[32];
                if (masked) form(std::true_type{}, 0);
                else form(std::false_type{}, 0);
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = f32_to_bf16x2(p[2 * j], p[2 * j + 1]);
                loaded(v[1]);
                store16(s_at, w);
                if (masked) form(std::true_type{}, 1);
                else form(std::false_type{}, 1);
#pragma unroll
                for (int j = 16; j < 32; ++j) w[j] = f32_to_bf16x2(p[2 * j], p[2 * j + 1]);
                store16(s_at + 16, w + 16);
                stored();
            }
            before_sync();
            arrive_warp(p_ready);
            arrive_warp(lse_empty);
            if (!(ok = wait.warp(delta_full, ph) && wait.warp(dp_full, ph))) break;
            after_sync();
            {
                float v[2][32];
                load32(d_at, v[0]);
                loaded(v[0]);
                load32(d_at + 32, v[1]);
                auto form = [&](int c, uint32_t* w) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 d = *reinterpret_cast<const float4*>(delta_s + half * 64 + c * 32 + j);
                        float x[4] = {v[c][j] - d.x, v[c][j + 1] - d.y, v[c][j + 2] - d.z, v[c][j + 3] - d.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            x[k] *= p[c * 32 + j + k];
                            if (masked && !(c * 32 + j + k >= f && c * 32 + j + k < e)) x[k] = 0.0f;   // (0 times what is not seen)
                        }
                        w[j / 2] = f32_to_bf16x2(x[0], x[1]);
                        w[j / 2 + 1] = f32_to_bf16x2(x[2], x[3]);
                    }
                };
                uint32_t w[16];
                form(0, w);
                loaded(v[1]);
                store16(d_at, w);
                form(1, w);
                store16(d_at + 16, w);
                stored();
            }
            before_sync();
            arrive_warp(ds_ready);
            arrive_warp(delta_empty);
        }
        // dV by the first half's warps, dK by the second's: a row a thread
        if (steps > 0) ok = ok && wait.warp(done, 0);
        after_sync();
        const bool nan = !ok || (steps > 0 && *gave_up), none = steps == 0;
        const uint32_t acc = (half ? dK : dV) + at;
        const float by = half ? g.scale : 1.0f;
        const long long row = (long long)t.k0 + t.first + r;
        if (a.parts > 1) {
            const long long width = (long long)kv_heads * g.head_dim;
            float* o = a.part + ((long long)(part * 2 + (half ? 0 : 1)) * g.k_rows + row) * width + (long long)kh * g.head_dim;
            if (!write_row<float, DP>(acc, o, r < keys, g.head_dim, g.head_dim % 4 == 0, by, nan, none)) *again = 1;
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
    if (*again && !*gave_up && warp < GR_COMPUTE) {
        float* const f = reinterpret_cast<float*>(smem);
        const int last = t.first + keys;
        for (; t.first < last; t.first += SA_B) {
            if (a.parts > 1) {
                const long long width = (long long)kv_heads * g.head_dim;
                float* const o = a.part + (long long)(part * 2) * g.k_rows * width;
                simt_grad_kv<__nv_bfloat16, DP, float>(g, t, kh, h0, h1, o, width, o + g.k_rows * width, width, f);
            } else {
                simt_grad_kv<__nv_bfloat16, DP, __nv_bfloat16>(g, t, kh, h0, h1, static_cast<__nv_bfloat16*>(g.dk), g.lddk,
                                                               static_cast<__nv_bfloat16*>(g.dv), g.lddv, f);
            }
            sa_sync();
        }
    }
}

template <int DP>
__global__ void __launch_bounds__(GR_THREADS, 1)
k_tc_grad_q(const __grid_constant__ GradMaps maps, const __grid_constant__ GradArgs a) {
    constexpr int TILE = GradTile<DP>::TILE;
    extern __shared__ unsigned char gr_smem_raw[];
    unsigned char* const smem = align1024(gr_smem_raw);
    unsigned char *const sq = smem, *const sd = sq + TILE, *const sk = sd + TILE, *const sv = sk + Q_K_STAGES * TILE;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(sv + Q_V_STAGES * TILE);
    const uint32_t bar = smem_u32(bars);
    const uint32_t q_full = bar, do_full = bar + 8, s_full = bar + 16 /* two */, dp_full = bar + 32, ds_ready = bar + 40,
                   done = bar + 48, rings = bar + 56;
    auto k_full = [&](int s) { return rings + 8u * s; };
    auto k_empty = [&](int s) { return rings + 8u * (Q_K_STAGES + s); };
    auto v_full = [&](int s) { return rings + 8u * (2 * Q_K_STAGES + s); };
    auto v_empty = [&](int s) { return rings + 8u * (2 * Q_K_STAGES + Q_V_STAGES + s); };
    constexpr int RINGS = 2 * (Q_K_STAGES + Q_V_STAGES);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(bars + 7 + RINGS);
    volatile int* const gave_up = reinterpret_cast<volatile int*>(slot + 1);
    volatile int* const again = gave_up + 1;           // a sum was not finite
    const AttnArgs& g = a.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.x % g.heads, kh = h / g.group;

    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / g.heads, ROWS, false, t)) return;
    const int rows = min(ROWS, t.nq - t.first);
    int lo, hi, unused;
    attn_keys_of(g, t, t.first, lo, unused);
    attn_keys_of(g, t, t.first + rows - 1, unused, hi);
    const int tile0 = lo / ROWS, steps = hi > lo ? (hi + ROWS - 1) / ROWS - tile0 : 0;

    if (threadIdx.x == 0) {
        for (uint32_t b : {q_full, do_full, s_full, s_full + 8, dp_full, done}) mbar_init(b, 1);
        mbar_init(ds_ready, GR_COMPUTE);
        for (int s = 0; s < RINGS; ++s) mbar_init(rings + 8u * s, 1);
        *gave_up = *again = 0;
        mbar_fence_init();
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
            load_tile<DP>(smem_u32(sq), &maps.q, h, t.q0 + t.first, q_full);
            int nk = 0, nv = 0;
            for (int n = 0; n < steps; ++n) {
                const int row = t.k0 + (tile0 + n) * ROWS, ks = nk % Q_K_STAGES, vs = nv % Q_V_STAGES;
                if (!wait(k_empty(ks), (uint32_t)(nk / Q_K_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sk) + ks * TILE, &maps.k, kh, row, k_full(ks));
                if (nk++ == 0) load_tile<DP>(smem_u32(sd), &maps.dout, h, t.q0 + t.first, do_full);
                if (!wait(v_empty(vs), (uint32_t)(nv / Q_V_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sv) + vs * TILE, &maps.v, kh, row, v_full(vs));
                ++nv;
            }
            wait.drain(q_full, 0);
            if (nk) wait.drain(do_full, 0);
            for (int i = max(0, nk - Q_K_STAGES); i < nk; ++i) wait.drain(k_full(i % Q_K_STAGES), (uint32_t)(i / Q_K_STAGES) & 1u);
            for (int i = max(0, nv - Q_V_STAGES); i < nv; ++i) wait.drain(v_full(i % Q_V_STAGES), (uint32_t)(i / Q_V_STAGES) & 1u);
        }
    } else if (warp == GR_COMPUTE + 1) {
        auto k_at = [&](int i) { return smem_u32(sk) + (uint32_t)(i % Q_K_STAGES) * TILE; };
        auto scores = [&](int i) {                                                 // S = Q K^T
            const int s = i % Q_K_STAGES;
            if (!wait.warp(k_full(s), (uint32_t)(i / Q_K_STAGES) & 1u)) return false;
            clear_rows<DP>(sk + s * TILE, t.nk - (tile0 + i) * ROWS);
            after_sync();
            if (lane == 0) {
                product_along<DP>(S + (i & 1) * 128, smem_u32(sq), k_at(i));
                commit(s_full + 8u * (i & 1));
            }
            __syncwarp();
            return true;
        };
        auto values = [&](int i) {                                                 // dP = dO V^T
            const int s = i % Q_V_STAGES;
            if (!wait.warp(v_full(s), (uint32_t)(i / Q_V_STAGES) & 1u)) return false;
            after_sync();
            if (lane == 0) {
                product_along<DP>(dP, smem_u32(sd), smem_u32(sv) + s * TILE);
                commit(dp_full);
                commit(v_empty(s));
            }
            __syncwarp();
            return true;
        };
        bool ok = steps > 0 && wait.warp(q_full, 0) && scores(0) && wait.warp(do_full, 0) && values(0) && (steps < 2 || scores(1));
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = wait.warp(ds_ready, (uint32_t)i & 1u))) break;
            if (i + 1 < steps && !(ok = values(i + 1))) break;                     // dP(i) has been read
            after_sync();
            if (lane == 0) {
                const uint32_t x = S + (i & 1) * 128;
                product_rows<DP>(dQ, x, x + 64, k_at(i), i > 0);
                commit(k_empty(i % Q_K_STAGES));
            }
            __syncwarp();
            if (i + 2 < steps && !(ok = scores(i + 2))) break;
        }
        if (lane == 0 && steps > 0) {
            commit(done);
            wait.drain(done, 0);
        }
    } else if (warp < GR_COMPUTE) {
        const int half = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t at = ((uint32_t)(warp & 3) * 32) << 16, d_at = dP + at + half * 64;
        int from, to;
        attn_keys_of(g, t, t.first + min(r, rows - 1), from, to);
        const long long stat = (long long)h * g.q_rows + t.q0 + t.first + min(r, rows - 1);
        const float lse2 = g.lse[stat] * LOG2E, delta = g.delta[stat];
        bool ok = true;
        for (int i = 0; i < steps; ++i) {
            const uint32_t s_at = S + (i & 1) * 128 + at + half * 64;
            const int k0 = (tile0 + i) * ROWS + half * 64;
            const int f = from - k0, e = to - k0;
            const bool masked = !__all_sync(0xFFFFFFFFu, f <= 0 && e >= 64);
            float p[64];
            if (!(ok = wait.warp(s_full + 8u * (i & 1), (uint32_t)(i >> 1) & 1u))) break;
            after_sync();
            {
                float v[2][32];
                load32(s_at, v[0]);
                loaded(v[0]);
                load32(s_at + 32, v[1]);
                auto form = [&](auto m, int c) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        p[c * 32 + j] = weight<decltype(m)::value>(v[c][j], a.scale2, lse2, c * 32 + j, f, e);
                };
                if (masked) form(std::true_type{}, 0);
                else form(std::false_type{}, 0);
                loaded(v[1]);
                if (masked) form(std::true_type{}, 1);
                else form(std::false_type{}, 1);
            }
            if (!(ok = wait.warp(dp_full, (uint32_t)i & 1u))) break;
            after_sync();
            {
                float v[2][32];
                load32(d_at, v[0]);
                loaded(v[0]);
                load32(d_at + 32, v[1]);
                auto form = [&](int c, uint32_t* w) {
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        float x = (v[c][j] - delta) * p[c * 32 + j], y = (v[c][j + 1] - delta) * p[c * 32 + j + 1];
                        if (masked) {                              // (0 times what is not seen)
                            if (!(c * 32 + j >= f && c * 32 + j < e)) x = 0.0f;
                            if (!(c * 32 + j + 1 >= f && c * 32 + j + 1 < e)) y = 0.0f;
                        }
                        w[j / 2] = f32_to_bf16x2(x, y);
                    }
                };
                uint32_t w[16];
                form(0, w);
                loaded(v[1]);
                store16(s_at, w);
                form(1, w);
                store16(s_at + 16, w);
                stored();
            }
            before_sync();
            arrive_warp(ds_ready);
        }
        if (steps > 0) ok = ok && wait.warp(done, 0);
        after_sync();
        // dQ: half of the columns by each half's warps
        const bool nan = !ok || (steps > 0 && *gave_up), none = steps == 0;
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(g.dq) + ((long long)t.q0 + t.first + r) * g.lddq + (long long)h * g.head_dim;
        if (!write_row<__nv_bfloat16, DP / 2>(dQ + at + half * (DP / 2), o + half * (DP / 2), r < rows,
                                              g.head_dim - half * (DP / 2), a.vec, g.scale, nan, none))
            *again = 1;
        before_sync();
    }
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        after_sync();
        free_all(tmem);
    }
    if (*again && !*gave_up && warp < GR_COMPUTE) {
        const int last = t.first + rows;
        for (; t.first < last; t.first += SA_B) {
            simt_grad_q<__nv_bfloat16, DP>(g, t, h, reinterpret_cast<float*>(smem));
            sa_sync();
        }
    }
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

template <typename K>
int tc_launch(K kernel, long long grid, int smem, const GradMaps& m, const GradArgs& a, cudaStream_t s) {
    if (grid > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return ISO_ERR_CUDA;
    TRAIN_LAUNCH((kernel<<<(unsigned)grid, GR_THREADS, smem, s>>>(m, a)));
    return ISO_OK;
}

template <int DP>
int launch_grad(const GradMaps& m, const GradArgs& a, cudaStream_t s) {
    const AttnArgs& g = a.g;
    if (g.k_rows)
        ISO_TRY(tc_launch(k_tc_grad_kv<DP>, attn_tiles(g.k_rows, g.n_seqs, ROWS) * (g.heads / g.group) * a.parts,
                          GradTile<DP>::KV_SMEM, m, a, s));
    if (g.q_rows)
        ISO_TRY(tc_launch(k_tc_grad_q<DP>, attn_tiles(g.q_rows, g.n_seqs, ROWS) * g.heads, GradTile<DP>::Q_SMEM, m, a, s));
    return ISO_OK;
}

}  // namespace

AttnGradPlan attn_grad_plan(long long q_rows, long long k_rows, const iso_attn_cfg& c) {
    (void)q_rows;
    const int group = c.heads / c.kv_heads;
    const long long items = (k_rows + ROWS - 1) / ROWS * c.kv_heads;
    AttnGradPlan p{1, 0};
    while (p.parts < group && items * p.parts < 8LL * train_sms()) ++p.parts;
    if (p.parts > 1) p.bytes = (size_t)p.parts * 2 * k_rows * c.kv_heads * c.head_dim * 4;
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
