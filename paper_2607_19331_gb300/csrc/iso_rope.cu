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
// as a binary32 number of half turns go to sincospif.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <cmath>

namespace iso {
namespace {

constexpr int ROPE_TPB = 256;
constexpr int ROPE_UNITS = 1024;      // units (of two 16-byte words in the vector form) a block takes
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

template <typename T>
__device__ __forceinline__ void rope_load(const T* p, float (&v)[8]) {
    Raw8<T> r;
    r.load(p);
    r.get(v);
}

// One unit of a head: VEC, eight pairs (of a head's turned part) or eight
// channels (of the rest), else one of either.
template <typename T, bool NEIGHBOURS, bool VEC>
__global__ void __launch_bounds__(ROPE_TPB) k_rope(const __grid_constant__ RopeArgs g) {
    extern __shared__ float2 rope_cs[];                  // [row][pair]: cosine, sine
    const int r0 = blockIdx.x * g.block_rows, rows = min(g.block_rows, g.rows - r0);
    for (int i = threadIdx.x; i < rows * g.pairs; i += ROPE_TPB) {
        const int r = i / g.pairs, p = i - r * g.pairs;
        const long long at = (long long)g.axis[p] * g.ldp + r0 + r;
        const long long pos = g.positions_i64 ? static_cast<const long long*>(g.positions)[at]
                                              : (long long)static_cast<const int*>(g.positions)[at];
        const unsigned long long a = (unsigned long long)pos * g.turns[p] + (1ULL << 31);
        float s, c;
        sincospif((float)(int)(a >> 32) * 0x1p-31f, &s, &c);
        rope_cs[i] = make_float2(c, g.inverse ? -s : s);
    }
    __syncthreads();
    constexpr int W = VEC ? 8 : 1;
    const int half = g.pairs, rot = 2 * g.pairs;
    const int turned = g.pairs / W, units = turned + (g.head_dim - rot) / W;   // units of a head
    const int per_row = units * g.heads;
    for (int i = threadIdx.x; i < rows * per_row; i += ROPE_TPB) {
        const int r = i / per_row, u = i - r * per_row, h = u / units, w = u - h * units;
        const T* x = static_cast<const T*>(g.x) + (long long)(r0 + r) * g.ldx + (long long)h * g.head_dim;
        T* y = static_cast<T*>(g.y) + (long long)(r0 + r) * g.ldy + (long long)h * g.head_dim;
        if (w >= turned) {
            const int c = rot + (w - turned) * W;
            if constexpr (VEC) {
                float v[8];
                rope_load(x + c, v);
                put8(y + c, v);
            } else {
                y[c] = x[c];
            }
            continue;
        }
        const float2* cs = rope_cs + r * g.pairs + w * W;
        if constexpr (VEC) {
            float a[8], b[8];
            if constexpr (NEIGHBOURS) {
                rope_load(x + w * 16, a);
                rope_load(x + w * 16 + 8, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = cs[j], q = cs[4 + j];
                    const float u0 = a[2 * j], w0 = a[2 * j + 1], u1 = b[2 * j], w1 = b[2 * j + 1];
                    a[2 * j] = u0 * t.x - w0 * t.y;
                    a[2 * j + 1] = u0 * t.y + w0 * t.x;
                    b[2 * j] = u1 * q.x - w1 * q.y;
                    b[2 * j + 1] = u1 * q.y + w1 * q.x;
                }
                put8(y + w * 16, a);
                put8(y + w * 16 + 8, b);
            } else {
                rope_load(x + w * 8, a);
                rope_load(x + half + w * 8, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 t = cs[j];
                    const float u0 = a[j], w0 = b[j];
                    a[j] = u0 * t.x - w0 * t.y;
                    b[j] = u0 * t.y + w0 * t.x;
                }
                put8(y + w * 8, a);
                put8(y + half + w * 8, b);
            }
        } else {
            const int ca = NEIGHBOURS ? 2 * w : w, cb = NEIGHBOURS ? 2 * w + 1 : half + w;
            const float2 t = cs[0];
            const float u0 = to_f32(x[ca]), w0 = to_f32(x[cb]);
            from_f32(u0 * t.x - w0 * t.y, y[ca]);
            from_f32(u0 * t.y + w0 * t.x, y[cb]);
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

template <typename T>
int launch_rope(const RopeArgs& g, bool neighbours, bool vec, cudaStream_t s) {
    const unsigned grid = (unsigned)((g.rows + g.block_rows - 1) / g.block_rows);
    const size_t smem = std::max<size_t>(1, (size_t)g.block_rows * g.pairs) * sizeof(float2);
    auto go = [&](auto nb, auto v) -> int {
        TRAIN_LAUNCH((k_rope<T, decltype(nb)::value, decltype(v)::value><<<grid, ROPE_TPB, smem, s>>>(g)));
        return ISO_OK;
    };
    if (neighbours) return vec ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    return vec ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
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
    // eight pairs a thread: their channels are whole 16-byte words of a head that
    // starts on such a boundary (in the halves form each half does)
    const bool vec = rows_aligned(x) && rows_aligned(y) && cfg->head_dim % 8 == 0 && pairs % 8 == 0;
    const long long units = (long long)g.heads * (vec ? (cfg->head_dim - pairs) / 8 : cfg->head_dim - pairs);
    g.block_rows = (int)std::max<long long>(1, std::min<long long>(ROPE_MAX_ROWS, ROPE_UNITS / std::max<long long>(1, units)));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return x->dtype == ISO_BF16 ? launch_rope<__nv_bfloat16>(g, cfg->neighbours, vec, s)
                                : launch_rope<float>(g, cfg->neighbours, vec, s);
}
