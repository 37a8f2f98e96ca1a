// iso_attn_fwd.cu -- attention on the fifth-generation tensor cores (bfloat16, head
// dimensions up to 128).
//
// A CTA has two tiles of 128 queries of one head and goes over their key tiles
// once:
//   S = Q K^T, m' = max(m, max S), P = exp2(c S - c m'), l <- l e + sum P,
//   O <- O e + P V,  e = exp2(c m - c m'),  c = scale log2 e,
// a row of a tile by one thread.  Scores, weights (bf16, over the scores that they
// came from) and sums stay in tensor memory, which the two tiles fill.  The tiles
// take turns: while the warps of one form its weights, the other's products
//   O_A(i) S_A(i+1) | O_B(i) S_B(i+1) | ...
// run.  The maximum is only moved when it grows by more than 2^RAISE (in the
// weights): until then e = 1, weights are up to 2^RAISE and the sums grow with
// them, which binary32 and bf16 hold as well; O is read and written back rarely.
// Measured: 8192 tokens, 28 heads over 4 of 128, causal, 392 us, 1.23 PFLOP/s (without
// causal 1.32).  What bounds it is a tile's chain: of 3600 clocks a step 1900 form the
// weights (960 of them exponentials, 512 at the least), the rest waits for two products
// and for the other tile's; sixteen warps with half a row a thread spill (899 us).
// Few queries over many keys: the key tiles are cut into parts for CTAs of their
// own, whose outputs, maxima and sums k_attn_join puts together.  (Not their
// log-sum-exps: those of large scores say nothing of the sums any more.)
#include "iso_attn.cuh"
#include "iso_attn_simt.cuh"
#include "iso_attn_tc.cuh"
#include "iso_tc.cuh"

#include <algorithm>

namespace iso {
namespace {

using namespace tc;

constexpr int FW_COMPUTE = 8;
constexpr int FW_THREADS = (FW_COMPUTE + 3) * 32;
constexpr int FW_K_STAGES = 2, FW_V_STAGES = 2;
constexpr int FW_ROWS = 2 * ROWS;
constexpr float RAISE = 8.0f;

struct FwdMaps {
    CUtensorMap q, k, v;
};
template <int DP>
struct FwdTile {
    static constexpr int TILE = DP / BOX * BOX_BYTES;
    static constexpr int SMEM = 1024 + (2 + FW_K_STAGES + FW_V_STAGES) * TILE + 256;
    static_assert(SMEM <= 232448, "shared memory of one CTA");
    static_assert(sa_smem<DP>(3, 1) <= (2 + FW_K_STAGES + FW_V_STAGES) * TILE, "the rows done over fit where the tiles were");
};
struct FwdArgs {
    AttnArgs g;
    uint64_t wait_ns;
    float scale2;                // scale log2 e
    int32_t vec;                 // rows of out start on 16-byte boundaries
    int32_t parts;               // parts of the key tiles
    float* part;                 // parts > 1: out as binary32, [part][q_rows][heads dim], then maxima and sums [part][heads][q_rows] each
};

// The key tiles [begin, end) of 128 queries from `first` on, those of a part
__device__ __forceinline__ void key_tiles(const FwdArgs& a, const AttnTile& t, int first, int rows, int part, int& begin, int& end) {
    begin = end = 0;
    if (rows <= 0) return;
    int lo, hi, unused;
    attn_keys_of(a.g, t, first, lo, unused);
    attn_keys_of(a.g, t, first + rows - 1, unused, hi);
    if (hi <= lo) return;
    const int t0 = lo / ROWS, n = (hi + ROWS - 1) / ROWS - t0;
    begin = t0 + (int)((long long)n * part / a.parts);
    end = t0 + (int)((long long)n * (part + 1) / a.parts);
}

// A CTA's rows done over in binary32 (iso_attn_simt.cuh), by 256 of its threads.
// Not inlined: nothing of it is held in registers before.
template <int DP>
__device__ __noinline__ void again_rows(const FwdArgs& a, float* smem) {
    const AttnArgs& g = a.g;
    const int part = blockIdx.x % a.parts, h = blockIdx.x / a.parts % g.heads;
    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / a.parts / g.heads, FW_ROWS, false, t)) return;
    const long long width = (long long)g.heads * g.head_dim;
    const int rows = min(FW_ROWS, t.nq - t.first), last = t.first + rows;
    for (int x = 0; x < 2; ++x) {
        int begin, end;
        key_tiles(a, t, t.first, min(ROWS, last - t.first), part, begin, end);
        for (const int stop = min(last, t.first + ROWS); t.first < stop; t.first += SA_B) {
            if (a.parts > 1) {
                float* const maxima = a.part + (long long)a.parts * g.q_rows * width + (long long)part * g.heads * g.q_rows;
                simt_attn<__nv_bfloat16, DP, float>(g, t, h, begin * ROWS, end * ROWS, a.part + (long long)part * g.q_rows * width, width,
                                                    maxima, smem, maxima + (long long)a.parts * g.heads * g.q_rows);
            } else
                simt_attn<__nv_bfloat16, DP, __nv_bfloat16>(g, t, h, begin * ROWS, end * ROWS, static_cast<__nv_bfloat16*>(const_cast<void*>(g.out)),
                                                            g.ldo, g.lse, smem);
            sa_sync();
        }
    }
}

template <int DP>
__global__ void __launch_bounds__(FW_THREADS, 1)
k_tc_attn(const __grid_constant__ FwdMaps maps, const __grid_constant__ FwdArgs a) {
    constexpr int TILE = FwdTile<DP>::TILE;
    extern __shared__ unsigned char fw_smem_raw[];
    unsigned char* const smem = align1024(fw_smem_raw);
    unsigned char *const sq = smem, *const sk = sq + 2 * TILE, *const sv = sk + FW_K_STAGES * TILE;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(sv + FW_V_STAGES * TILE);
    const uint32_t bar = smem_u32(bars);
    // of the two tiles: scores there, weights there, sums there, queries there
    auto s_full = [&](int x) { return bar + 8u * x; };
    auto p_ready = [&](int x) { return bar + 16u + 8u * x; };
    auto o_done = [&](int x) { return bar + 32u + 8u * x; };
    auto q_full = [&](int x) { return bar + 48u + 8u * x; };
    const uint32_t done = bar + 64 /* two */, cleared = bar + 80, rings = bar + 88;
    auto k_full = [&](int s) { return rings + 8u * s; };
    auto k_empty = [&](int s) { return rings + 8u * (FW_K_STAGES + s); };
    auto v_full = [&](int s) { return rings + 8u * (2 * FW_K_STAGES + s); };
    auto v_empty = [&](int s) { return rings + 8u * (2 * FW_K_STAGES + FW_V_STAGES + s); };
    constexpr int RINGS = 2 * (FW_K_STAGES + FW_V_STAGES);
    uint32_t* const slot = reinterpret_cast<uint32_t*>(bars + 11 + RINGS);
    volatile int* const gave_up = reinterpret_cast<volatile int*>(slot + 1);
    volatile int* const again = gave_up + 1;           // a sum was not finite
    const AttnArgs& g = a.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = blockIdx.x % a.parts, h = blockIdx.x / a.parts % g.heads, kh = h / g.group;

    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / a.parts / g.heads, FW_ROWS, false, t)) return;
    const int rows = min(FW_ROWS, t.nq - t.first);
    int begin[2], end[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) key_tiles(a, t, t.first + x * ROWS, min(ROWS, rows - x * ROWS), part, begin[x], end[x]);
    // the tiles that either needs
    const bool has[2] = {end[0] > begin[0], end[1] > begin[1]};
    const int u0 = has[0] && has[1] ? min(begin[0], begin[1]) : has[0] ? begin[0] : begin[1];
    const int u1 = has[0] && has[1] ? max(end[0], end[1]) : has[0] ? end[0] : end[1];
    const int steps = u1 - u0;

    if (warp == FW_COMPUTE && lane == 0) {
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(p_ready(x), FW_COMPUTE / 2);
            mbar_init(o_done(x), 1);
            mbar_init(q_full(x), 1);
        }
        mbar_init(done, 1);
        mbar_init(done + 8, 1);
        mbar_init(cleared, 1);
        for (int s = 0; s < FW_K_STAGES; ++s) {
            mbar_init(k_full(s), 1);
            mbar_init(k_empty(s), 2);            // both tiles' products
        }
        for (int s = 0; s < FW_V_STAGES; ++s) {
            mbar_init(v_full(s), 1);
            mbar_init(v_empty(s), 2);
        }
        *gave_up = *again = 0;
        mbar_fence_init();
        if (steps > 0) {                         // the first copies, while the CTA gets ready
            for (int x = 0; x < 2; ++x)
                if (has[x]) load_tile<DP>(smem_u32(sq) + x * TILE, &maps.q, h, t.q0 + t.first + x * ROWS, q_full(x));
            load_tile<DP>(smem_u32(sk), &maps.k, kh, t.k0 + u0 * ROWS, k_full(0));
            load_tile<DP>(smem_u32(sv), &maps.v, kh, t.k0 + u0 * ROWS, v_full(0));
        }
    }
    if (warp == 0) alloc_all(smem_u32(slot));
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(slot);
    const Waits wait = {a.wait_ns, gave_up};
    auto S = [&](int x) { return tmem + 128u * x; };
    auto O = [&](int x) { return tmem + 256u + 128u * x; };

    if (warp == FW_COMPUTE) {
        // copies, of the second key tile on
        if (lane == 0 && steps > 0) {
            int nk = 1, nv = 1;
            for (int i = 1; i < steps; ++i) {
                const int row = t.k0 + (u0 + i) * ROWS, ks = nk % FW_K_STAGES, vs = nv % FW_V_STAGES;
                if (!wait(k_empty(ks), (uint32_t)(nk / FW_K_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sk) + ks * TILE, &maps.k, kh, row, k_full(ks));
                ++nk;
                if (!wait(v_empty(vs), (uint32_t)(nv / FW_V_STAGES + 1) & 1u)) break;
                load_tile<DP>(smem_u32(sv) + vs * TILE, &maps.v, kh, row, v_full(vs));
                ++nv;
            }
            // no copy is in flight when the CTA ends, after a give-up either
            for (int x = 0; x < 2; ++x)
                if (has[x]) wait.drain(q_full(x), 0);
            for (int i = max(0, nk - FW_K_STAGES); i < nk; ++i) wait.drain(k_full(i % FW_K_STAGES), (uint32_t)(i / FW_K_STAGES) & 1u);
            for (int i = max(0, nv - FW_V_STAGES); i < nv; ++i) wait.drain(v_full(i % FW_V_STAGES), (uint32_t)(i / FW_V_STAGES) & 1u);
        }
    } else if (warp > FW_COMPUTE) {
        // products, a warp for either tile: O(i), then S(i + 1) over its weights.  (The
        // whole warp waits and clears, one lane issues.)
        const int x = warp - FW_COMPUTE - 1;
        Slot<FW_K_STAGES> ks;                        // K of the next scores
        Slot<FW_V_STAGES> vs;
        const uint32_t q_s = smem_u32(sq) + (uint32_t)x * TILE, k_s = smem_u32(sk), v_s = smem_u32(sv);
        auto in = [&](int i) { return u0 + i >= begin[x] && u0 + i < end[x]; };
        auto scores = [&](int i) {                                                 // S = Q K^T
            if (!wait.warp(k_full(ks.at), ks.parity)) return false;
            after_sync();
            if (elected()) {
                if (in(i)) {
                    product_along<DP>(S(x), q_s, k_s + (uint32_t)ks.at * TILE);
                    commit(s_full(x));
                }
                commit(k_empty(ks.at));
            }
            __syncwarp();
            ks.next();
            return true;
        };
        bool ok = steps > 0 && (!has[x] || wait.warp(q_full(x), 0)) && scores(0);
        for (int i = 0; ok && i < steps; ++i) {
            if (!(ok = wait.warp(v_full(vs.at), vs.parity))) break;
            if (in(i)) {
                const int j = u0 + i - begin[x];
                if (i == steps - 1) {
                    // one warp clears the rows behind the sequence's end, for both
                    if (x == 0 || !has[0] || u0 + i >= end[0]) clear_rows<DP>(sv + vs.at * TILE, t.nk - (u0 + i) * ROWS);
                    else if (!(ok = wait.warp(cleared, 0))) break;
                    if (x == 0) arrive_warp(cleared);
                }
                if (!(ok = wait.warp(p_ready(x), (uint32_t)j & 1u))) break;
                after_sync();
                if (elected()) {
                    product_rows<DP, 128>(O(x), S(x), v_s + (uint32_t)vs.at * TILE, j > 0);   // O += P V
                    commit(o_done(x));
                }
                __syncwarp();
            }
            if (elected()) commit(v_empty(vs.at));
            __syncwarp();
            vs.next();
            if (i + 1 < steps) ok = scores(i + 1);
        }
        // no product runs on when the tensor memory is freed, after a give-up either
        if (steps > 0 && elected()) {
            commit(done + 8u * x);
            wait.drain(done + 8u * x, 0);
        }
    } else {
        const int x = warp >> 2, r = (warp & 3) * 32 + lane, mine = min(ROWS, rows - x * ROWS);
        const int first = t.first + x * ROWS, n = end[x] - begin[x];
        const uint32_t at = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t s_at = S(x) + at, o_at = O(x) + at;
        int from = 0, to = 0;
        if (mine > 0) attn_keys_of(g, t, first + min(r, mine - 1), from, to);
        const float c = a.scale2;
        float m = -INFINITY, l = 0.0f;
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const int k0 = (begin[x] + j) * ROWS, f = from - k0, e = to - k0;
            const bool masked = !__all_sync(0xFFFFFFFFu, f <= 0 && e >= ROWS);
            if (!(ok = wait.warp(s_full(x), (uint32_t)j & 1u))) break;
            after_sync();
            float v[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q) load32(s_at + q * 32, v[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q) loaded(v[q]);
            if (masked) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(q * 32 + i >= f && q * 32 + i < e)) v[q][i] = -INFINITY;
            }
            float tops[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                tops[q] = max3(v[q][0], v[q][1], v[q][2]);
#pragma unroll
                for (int i = 3; i < 31; i += 2) tops[q] = max3(tops[q], v[q][i], v[q][i + 1]);
                tops[q] = fmaxf(tops[q], v[q][31]);
            }
            const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
            // from -Inf any finite maximum is a raise
            const bool raise = (top - m) * c > RAISE;
            if (__any_sync(0xFFFFFFFFu, raise)) {
                const float by = raise ? ex2((m - top) * c) : 1.0f;
                if (raise) m = top;
                l *= by;
                if (j > 0) {
                    if (!(ok = wait.warp(o_done(x), (uint32_t)(j - 1) & 1u))) break;
                    after_sync();
#pragma unroll 1
                    for (int q = 0; q < DP; q += 32) {
                        float o[32];
                        load32(o_at + q, o);
                        loaded(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] *= by;
                        store32(o_at + q, o);
                    }
                }
            }
            const float base = m == -INFINITY ? 0.0f : -m * c;
            const uint64_t cc = pair_of(c, c), bb = pair_of(base, base);
            uint64_t sum[2] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    float p0, p1;
                    parts_of(fma2(pair_of(v[q][i], v[q][i + 1]), cc, bb), p0, p1);
                    p0 = ex2(p0);
                    p1 = ex2(p1);
                    sum[i / 2 % 2] = add2(sum[i / 2 % 2], pair_of(p0, p1));
                    w[i / 2] = f32_to_bf16x2(p0, p1);
                }
                store16(s_at + q * 16, w);
            }
            stored();
            before_sync();
            arrive_warp(p_ready(x));
            float l0, l1;
            parts_of(add2(sum[0], sum[1]), l0, l1);
            l += l0 + l1;
        }
        if (n > 0) ok = ok && wait.warp(o_done(x), (uint32_t)(n - 1) & 1u);
        after_sync();
        const bool nan = !ok, none = n == 0;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l, lse = nan ? __int_as_float(0x7FFFFFFF) : m * g.scale + logf(l);
        const long long row = (long long)t.q0 + first + r, width = (long long)g.heads * g.head_dim;
        bool finite;
        if (a.parts > 1) {
            float* o = a.part + ((long long)part * g.q_rows + row) * width + (long long)h * g.head_dim;
            finite = write_row<float, DP>(o_at, o, r < mine, g.head_dim, true, inv, nan, none);
            if (r < mine) {
                float* const maxima = a.part + (long long)a.parts * g.q_rows * width + ((long long)part * g.heads + h) * g.q_rows + row;
                maxima[0] = nan ? lse : m * g.scale;
                // (without the rounding of m c, which is in every weight)
                maxima[(long long)a.parts * g.heads * g.q_rows] = m == -INFINITY ? 0.0f : l * ex2(-fmaf(m, c, -__fmul_rn(m, c)));
            }
        } else {
            __nv_bfloat16* o = static_cast<__nv_bfloat16*>(const_cast<void*>(g.out)) + row * g.ldo + (long long)h * g.head_dim;
            finite = write_row<__nv_bfloat16, DP>(o_at, o, r < mine, g.head_dim, a.vec, inv, nan, none);
            if (r < mine) g.lse[(long long)h * g.q_rows + row] = lse;
        }
        // l counts the row's largest weight, 1 or more, times 2 to the rounding of m c: with
        // scores of 1e9 and beyond that is any power, and what it leaves of l no sum
        if (!finite || (r < mine && m > -INFINITY && !(l > 0.25f && l < 0x1p100f))) *again = 1;
        before_sync();
    }
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        after_sync();
        free_all(tmem);
    }
    if (*again && !*gave_up && warp < SA_TPB / 32) again_rows<DP>(a, reinterpret_cast<float*>(smem));
}

// The parts of a row of one head put together: with m the largest m_p, l = sum l_p
// e^(m_p - m), lse = m + log l, out = sum l_p e^(m_p - m) out_p / l.  Eight columns a thread.
template <bool VEC>
__global__ void __launch_bounds__(256) k_attn_join(const __grid_constant__ FwdArgs a) {
    const AttnArgs& g = a.g;
    const int segs = g.head_dim / 8;
    const long long width = (long long)g.heads * g.head_dim;
    int first = 0, last = g.q_rows;
    if (g.n_seqs) {
        first = min(max(g.q_ends[0], 0), g.q_rows);
        last = min(max(g.q_ends[g.n_seqs], 0), g.q_rows);
    }
    const long long n = (long long)max(last - first, 0) * g.heads * segs;
    const float* maxima = a.part + (long long)a.parts * g.q_rows * width;
    const float* sums = maxima + (long long)a.parts * g.heads * g.q_rows;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const int s = (int)(i % segs), h = (int)(i / segs % g.heads);
        const long long row = first + i / segs / g.heads;
        float m = -INFINITY, sum = 0.0f, acc[8] = {};
#pragma unroll 8
        for (int p = 0; p < a.parts; ++p) m = fmaxf(m, maxima[((long long)p * g.heads + h) * g.q_rows + row]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
        for (int p = 0; p < a.parts; ++p) {
            const long long at = ((long long)p * g.heads + h) * g.q_rows + row;
            const float w = sums[at] * expf(maxima[at] - base);
            sum += w;
            float x[8];                          // (of a part without a seen key: zeros, of weight 0)
            load8<true>(a.part + ((long long)p * g.q_rows + row) * width + (long long)h * g.head_dim, s * 8, g.head_dim, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = fmaf(w, x[j], acc[j]);
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] *= inv;
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(const_cast<void*>(g.out)) + row * g.ldo + (long long)h * g.head_dim;
        store8<VEC>(o, s * 8, g.head_dim, acc);
        if (s == 0) g.lse[(long long)h * g.q_rows + row] = m + logf(sum);
    }
}

template <int DP>
int launch_attn(const FwdMaps& m, const FwdArgs& a, cudaStream_t s) {
    const AttnArgs& g = a.g;
    const long long grid = attn_tiles(g.q_rows, g.n_seqs, FW_ROWS) * g.heads * a.parts;
    if (grid > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> done{0};
    ISO_TRY(allow_smem(k_tc_attn<DP>, FwdTile<DP>::SMEM, done));
    TRAIN_LAUNCH((k_tc_attn<DP><<<(unsigned)grid, FW_THREADS, FwdTile<DP>::SMEM, s>>>(m, a)));
    return ISO_OK;
}

}  // namespace

AttnPlan attn_plan(long long q_rows, long long k_rows, const iso_attn_cfg& c) {
    const long long items = attn_tiles(q_rows, c.n_seqs, FW_ROWS) * c.heads;
    const long long tiles = k_rows / std::max(1, c.n_seqs) / ROWS;       // of a sequence, on average
    AttnPlan p{1, 0};
    // CTAs for every SM, two key tiles or more in each (one token over 4096 keys, 12 heads over 2: 21 us,
    // in one part 47; over 65536 keys, 28 over 4: 150, 668; over 1024 keys, 12 over 2: 16, 17)
    p.parts = (int)std::max<long long>(1, std::min<long long>({train_sms() / std::max<long long>(1, items), tiles / 2, 64}));
    if (p.parts > 1) p.bytes = (size_t)p.parts * q_rows * c.heads * (c.head_dim + 2) * 4;
    return p;
}

int attn_tc(const AttnArgs& g, const AttnPlan& p, float* part, cudaStream_t s) {
    FwdMaps m;
    ISO_TRY(head_map(&m.q, g.q, g.q_rows, g.heads, g.head_dim, g.ldq));
    ISO_TRY(head_map(&m.k, g.k, g.k_rows, g.heads / g.group, g.head_dim, g.ldk));
    ISO_TRY(head_map(&m.v, g.v, g.k_rows, g.heads / g.group, g.head_dim, g.ldv));
    FwdArgs a{};
    a.g = g;
    a.wait_ns = attn_wait_ns();
    a.scale2 = g.scale * LOG2E;
    a.vec = (reinterpret_cast<uintptr_t>(g.out) & 15u) == 0 && g.ldo % 8 == 0;
    a.parts = p.parts;
    a.part = part;
    ISO_TRY(g.head_dim <= 64 ? launch_attn<64>(m, a, s) : launch_attn<128>(m, a, s));
    if (p.parts == 1) return ISO_OK;
    const long long n = (long long)g.q_rows * g.heads * (g.head_dim / 8);
    const unsigned grid = (unsigned)std::min<long long>((n + 255) / 256, 1 << 20);
    TRAIN_LAUNCH((a.vec ? k_attn_join<true><<<grid, 256, 0, s>>>(a) : k_attn_join<false><<<grid, 256, 0, s>>>(a)));
    return ISO_OK;
}

}  // namespace iso
