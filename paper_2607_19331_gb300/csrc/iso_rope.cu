// iso_rope.cu -- rotary positions with several axes, and their gradient (the
// turn back).
//
// A row is read once and written once, 4 bytes an entry in bf16, against one
// sine and cosine per pair of channels and row, shared by all heads: bound by
// HBM.  So a block takes a few rows: it forms the sines and cosines of its rows in
// shared memory and then turns all their heads.
//
// Angles.  freq * p as a binary32 product would be wrong by p 2^-24 radians (0.006
// at position 100000), so the angle is a fixed-point fraction of a whole turn:
// F = freq / (2 pi) mod 1 as a 64-bit integer, formed on the host, and p F mod
// 2^64 is the angle mod one turn, exactly, for any 64-bit p.  Its upper 32 bits
// as a binary32 number of half turns, off by 2^-26 turns at most, go to sincospif.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <cmath>

namespace iso {
namespace {

// 64: 91 us there and back over 16384 x 4096 bf16, 128: 100, 256: 109 (binary32: 168, 164, 161)
constexpr int ROPE_TPB = 64;
// units in flight a thread: 64 bytes of loads (twice that: 107 us)
template <typename T>
constexpr int rope_each(int u) { return u == 1 ? 4 : 16 / (u * (int)sizeof(T) / 2); }
constexpr int ROPE_MAX_ROWS = 16;

struct RopeArgs {
    unsigned long long turns[ISO_ROPE_MAX_PAIRS];
    uint8_t axis[ISO_ROPE_MAX_PAIRS];
    const void* x;
    void* y;
    const void* positions;
    long long ldx, ldy, ldp;
    int32_t rows, heads, head_dim, pairs;
    int32_t positions_i64, inverse, block_rows;
};

// sines and cosines of the block's rows, [row][pair]
__device__ __forceinline__ void rope_angles(const RopeArgs& g, float2* cs, int r0, int rows) {
    for (int i = threadIdx.x; i < rows * g.pairs; i += ROPE_TPB) {
        const int r = i / g.pairs, p = i - r * g.pairs;
        const long long at = (long long)g.axis[p] * g.ldp + r0 + r;
        const long long pos = g.positions_i64 ? static_cast<const long long*>(g.positions)[at]
                                              : (long long)static_cast<const int*>(g.positions)[at];
        const unsigned long long a = (unsigned long long)pos * g.turns[p] + (1ULL << 31);
        float s, c;
        sincospif((float)(int)(a >> 32) * 0x1p-31f, &s, &c);
        cs[i] = make_float2(c, g.inverse ? -s : s);
    }
}

// U channels of a row, side by side: four in 8 or 16 bytes, or one
template <typename T, int U>
struct Run;
template <>
struct Run<float, 4> {
    float4 x;
    __device__ __forceinline__ void load(const float* p) { x = __ldcs(reinterpret_cast<const float4*>(p)); }
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
    static __device__ __forceinline__ void put(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <>
struct Run<__nv_bfloat16, 4> {
    uint2 x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = __ldcs(reinterpret_cast<const uint2*>(p)); }
    __device__ __forceinline__ void get(float (&v)[4]) const {
        bf16x2_to_f32(x.x, v[0], v[1]);
        bf16x2_to_f32(x.y, v[2], v[3]);
    }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, const float (&v)[4]) {
        *reinterpret_cast<uint2*>(p) = make_uint2(f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3]));
    }
};
template <typename T>
struct Run<T, 1> {
    T x;
    __device__ __forceinline__ void load(const T* p) { x = *p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32(x); }
    static __device__ __forceinline__ void put(T* p, const float (&v)[1]) { from_f32(v[0], *p); }
};

// (u, w) turned, in the same operations for every unit, so that a row's bits do not
// depend on how it lies
__device__ __forceinline__ void turn(float& u, float& w, float c, float s) {
    const float a = __fmaf_rn(u, c, -__fmul_rn(w, s)), b = __fmaf_rn(u, s, __fmul_rn(w, c));
    u = a;
    w = b;
}

// A unit is U pairs (two runs of channels, from either half or side by side) or one
// run of the channels that are copied.  A thread goes through the block's units in steps of
// the block, by additions; its first ones are loaded before the angles are formed.
template <typename T, bool NEIGHBOURS, int U>
__global__ void __launch_bounds__(ROPE_TPB) k_rope(const __grid_constant__ RopeArgs g) {
    extern __shared__ float2 rope_cs[];
    constexpr int EACH = rope_each<T>(U);
    const int r0 = blockIdx.x * g.block_rows, rows = min(g.block_rows, g.rows - r0);
    const int turned = g.pairs / U, units = turned + (g.head_dim - 2 * g.pairs) / U;
    const int step_h = ROPE_TPB / units, step_w = ROPE_TPB - step_h * units;
    int r = 0, h = (int)threadIdx.x / units, w = (int)threadIdx.x - h * units;
    auto settle = [&] {
        while (h >= g.heads && r < rows) {
            h -= g.heads;
            ++r;
        }
    };
    settle();
    // a unit's runs of channels
    auto first = [&](int unit) {
        return unit >= turned ? 2 * g.pairs + (unit - turned) * U : NEIGHBOURS ? unit * 2 * U : unit * U;
    };
    auto second = [&](int unit) { return NEIGHBOURS ? unit * 2 * U + U : g.pairs + unit * U; };
    bool formed = false;
    for (;;) {
        Run<T, U> a[EACH], b[EACH];
        int rr[EACH], hh[EACH], ww[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            rr[k] = r;
            hh[k] = h;
            ww[k] = w;
            if (r < rows) {
                const T* x = static_cast<const T*>(g.x) + (long long)(r0 + r) * g.ldx + (long long)h * g.head_dim;
                a[k].load(x + first(w));
                if (w < turned) b[k].load(x + second(w));
                h += step_h;
                w += step_w;
                if (w >= units) {
                    w -= units;
                    ++h;
                }
                settle();
            }
        }
        if (!formed) {
            rope_angles(g, rope_cs, r0, rows);
            __syncthreads();
            formed = true;
        }
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (rr[k] >= rows) return;
            T* y = static_cast<T*>(g.y) + (long long)(r0 + rr[k]) * g.ldy + (long long)hh[k] * g.head_dim;
            float u[U], v[U];
            a[k].get(u);
            if (ww[k] < turned) {
                b[k].get(v);
                const float2* cs = rope_cs + rr[k] * g.pairs + ww[k] * U;
                if constexpr (U == 1) {
                    turn(u[0], v[0], cs[0].x, cs[0].y);
                } else {
#pragma unroll
                    for (int j = 0; j < U / 2; ++j) {
                        const float4 t = reinterpret_cast<const float4*>(cs)[j];           // two pairs
                        if constexpr (NEIGHBOURS) {
                            float* const z = j == 0 ? u : v;
                            turn(z[0], z[1], t.x, t.y);
                            turn(z[2], z[3], t.z, t.w);
                        } else {
                            turn(u[2 * j], v[2 * j], t.x, t.y);
                            turn(u[2 * j + 1], v[2 * j + 1], t.z, t.w);
                        }
                    }
                }
                Run<T, U>::put(y + second(ww[k]), v);
            }
            Run<T, U>::put(y + first(ww[k]), u);
        }
    }
}

// t modulo 1 as a 64-bit fraction of one
unsigned long long fraction(double t) {
    t = std::ldexp(t - std::rint(t), 32);                     // exact
    const double h = std::trunc(t), l = std::rint(std::ldexp(t - h, 32));
    return ((unsigned long long)(long long)h << 32) + (unsigned long long)(long long)l;
}
// freq / (2 pi) modulo 1, with 1 / (2 pi) as the sum of two binary64 numbers: the
// product of the first one as a rounded value and its exact error
unsigned long long fixed_turns(double freq) {
    const double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57, t = freq * hi;
    return fraction(t) + fraction(std::fma(freq, hi, -t) + freq * lo);
}

template <typename T, int U>
int launch_rope(RopeArgs& g, bool neighbours, cudaStream_t s) {
    const long long units = (long long)g.heads * ((g.head_dim - g.pairs) / U);
    g.block_rows = (int)std::max<long long>(1, std::min<long long>(ROPE_MAX_ROWS, ROPE_TPB * rope_each<T>(U) / std::max<long long>(1, units)));
    const unsigned grid = (unsigned)((g.rows + g.block_rows - 1) / g.block_rows);
    const size_t smem = std::max<size_t>(1, (size_t)g.block_rows * g.pairs) * sizeof(float2);
    TRAIN_LAUNCH((neighbours ? k_rope<T, true, U><<<grid, ROPE_TPB, smem, s>>>(g) : k_rope<T, false, U><<<grid, ROPE_TPB, smem, s>>>(g)));
    return ISO_OK;
}
// Four pairs a unit where their runs of channels are whole loads in every head of
// every row, else one (16384 x 4096 bf16, one way: 46 us; eight pairs 51, one 102)
template <typename T>
int launch_rope(RopeArgs& g, bool neighbours, cudaStream_t s) {
    constexpr uint64_t bytes = 4 * sizeof(T);
    const bool four = g.pairs % 4 == 0 && g.head_dim % 4 == 0 && (reinterpret_cast<uintptr_t>(g.x) | reinterpret_cast<uintptr_t>(g.y)) % bytes == 0 &&
                      (g.rows == 1 || (g.ldx * sizeof(T) % bytes == 0 && g.ldy * sizeof(T) % bytes == 0));
    return four ? launch_rope<T, 4>(g, neighbours, s) : launch_rope<T, 1>(g, neighbours, s);
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" int32_t iso_rope(const iso_mat* x, const void* positions, int32_t positions_i64, int64_t ld_positions,
                            const iso_rope_cfg* cfg, const iso_mat* y, void* stream) {
    ISO_TRY(check_mat(x));
    ISO_TRY(check_mat(y));
    if (!cfg || cfg->reserved != 0 || cfg->head_dim < 1 || cfg->axes < 1 || cfg->axes > ISO_ROPE_MAX_AXES ||
        (cfg->neighbours != 0 && cfg->neighbours != 1) || (cfg->inverse != 0 && cfg->inverse != 1) ||
        (positions_i64 != 0 && positions_i64 != 1))
        return ISO_ERR_ARG;
    if (cfg->rot_dim < 0 || cfg->rot_dim % 2 || cfg->rot_dim > cfg->head_dim || cfg->rot_dim > 2 * ISO_ROPE_MAX_PAIRS)
        return ISO_ERR_ARG;
    const int pairs = cfg->rot_dim / 2;
    if (pairs && (!cfg->freq || !cfg->axis)) return ISO_ERR_ARG;
    RopeArgs g{};
    for (int i = 0; i < pairs; ++i) {
        if (!std::isfinite(cfg->freq[i]) || cfg->axis[i] < 0 || cfg->axis[i] >= cfg->axes) return ISO_ERR_ARG;
        g.turns[i] = fixed_turns(cfg->freq[i]);
        g.axis[i] = (uint8_t)cfg->axis[i];
    }
    if (x->rows != y->rows || x->cols != y->cols || x->cols % cfg->head_dim) return ISO_ERR_SHAPE;
    if (x->dtype != y->dtype) return ISO_ERR_DTYPE;
    if (ld_positions < x->rows) return ISO_ERR_SHAPE;
    if (ld_positions > STRIDE_LIMIT) return ISO_ERR_UNSUPPORTED;
    if (x->rows == 0 || x->cols == 0) return ISO_OK;
    const int pos_size = positions_i64 ? 8 : 4;
    if (!positions) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(positions) % pos_size) return ISO_ERR_ALIGN;
    const bool same = x->data == y->data && (x->ld == y->ld || x->rows == 1);
    const Bytes2D pb = {reinterpret_cast<uintptr_t>(positions), (uint64_t)cfg->axes, (uint64_t)x->rows * pos_size,
                        (uint64_t)ld_positions * pos_size};
    if ((!same && share_bytes(bytes_of(x), bytes_of(y))) || share_bytes(pb, bytes_of(y))) return ISO_ERR_ARG;
    g.x = x->data;
    g.y = y->data;
    g.positions = positions;
    g.ldx = x->ld;
    g.ldy = y->ld;
    g.ldp = ld_positions;
    g.rows = (int)x->rows;
    g.heads = (int)(x->cols / cfg->head_dim);
    g.head_dim = cfg->head_dim;
    g.pairs = pairs;
    g.positions_i64 = positions_i64;
    g.inverse = cfg->inverse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return x->dtype == ISO_BF16 ? launch_rope<__nv_bfloat16>(g, cfg->neighbours, s)
                                : launch_rope<float>(g, cfg->neighbours, s);
}
