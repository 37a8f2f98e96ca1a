// iso_act.cu -- 8-bit activation checkpoints: pack, unpack, and the SwiGLU
// activation with its gradients through checkpoints (formats and formulas in
// include/iso.h).
//
// All four are one pass over their operands and bound by HBM: a few integer
// and binary32 operations per entry.  A warp takes 256 channels of one row at
// a time, eight per lane, so a group of 32 channels is four neighbouring lanes
// and its maximum two shuffles; loads are 16 bytes per lane and a warp's codes
// 256 contiguous bytes.
#include "iso_train.cuh"

#include <algorithm>
#include <atomic>

namespace iso {

int train_sms() {
    static std::atomic<int> sms[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
    int n = sms[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 152;
        sms[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

namespace {

constexpr int ACT_TPB = 128;
constexpr int ACT_WPB = ACT_TPB / 32;
// k_swiglu_pack on binary32, 8192 x 8960: 177 us with 256 threads a block, 204 us with 128
constexpr int SWIGLU_F32_TPB = 256;

struct ActView {
    uint8_t* codes;
    uint8_t* exps;
    long long ld_codes, ld_exps;
};

// Runs of SEGS neighbouring segments of a row, row after row: item i is run
// i % runs of row i / runs.
struct Items {
    long long n;
    int runs;
};

// this lane's eight codes at channel c (below the padded width) and the
// group's exponent byte; the last group's lanes also fill the exponent padding
__device__ __forceinline__ void act_store(const ActView& a, long long row, int c, int cols, uint2 codes, uint32_t b) {
    const int padded = (cols + ISO_ACT_GROUP - 1) & ~(ISO_ACT_GROUP - 1);
    if (c >= padded) return;
    *reinterpret_cast<uint2*>(a.codes + row * a.ld_codes + c) = codes;
    if ((c & (ISO_ACT_GROUP - 1)) == 0) {
        uint8_t* e = a.exps + row * a.ld_exps;
        const int g = c / ISO_ACT_GROUP, groups = padded / ISO_ACT_GROUP;
        e[g] = (uint8_t)b;
        if (g == groups - 1)
            for (int p = groups; p < ((groups + 7) & ~7); ++p) e[p] = 1;
    }
}

__device__ __forceinline__ void act_load(const ActView& a, long long row, int c, int cols, uint2& codes, uint32_t& b) {
    codes = make_uint2(0u, 0u);
    b = 1;
    if (c < cols) {
        codes = __ldcs(reinterpret_cast<const uint2*>(a.codes + row * a.ld_codes + c));
        b = a.exps[row * a.ld_exps + c / ISO_ACT_GROUP];
    }
}

// Four segments of a row to a warp: their addresses are one base and constant
// offsets, and their loads are all in flight before the first is used.  The
// issue rate is as near a bound as HBM: with one segment a warp and a
// persistent grid the packing took 21 instructions an entry and 110 us for
// 16384 x 8960 bf16, the SwiGLU pair 322 + 352 us for 8192 x 18944.
// Blocks are small and not persistent, so that those in flight cover one moving
// window of every operand: blocks of 128 threads measured 74 / 69 / 203 / 248 us
// (pack, unpack, SwiGLU, its gradients at those sizes: 6.0, 6.4, 6.2, 6.3 TB/s),
// of 256 threads 78 / 69 / 228 / 253 us, a persistent grid 76 / 74 / 221 / 246 us.
constexpr int SEGS = 4;

// One run of a warp: row, first channel of this lane, and how many of its
// segments lie wholly inside rows that start on 16-byte boundaries (those take
// the fast form; the others check every entry).
struct Run {
    long long row;
    int c, full;
    __device__ __forceinline__ Run(const Items& it, long long i, int lane, int cols, bool vec) {
        row = i / it.runs;
        const int c0 = (int)(i - row * it.runs) * (SEGS * TRAIN_SEG);
        c = c0 + lane * 8;
        full = vec ? min(SEGS, (cols - c0) / TRAIN_SEG) : 0;
    }
};
#define ACT_FOR_RUNS                                                                          \
    const int lane = threadIdx.x & 31;                                                        \
    for (long long i = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < it.n; \
         i += (long long)gridDim.x * (blockDim.x >> 5))

// Exponent bytes of a run's full segments: every lane of a group holds all
// four, and stores the one of its place in the group.
__device__ __forceinline__ void store_exps(const ActView& a, const Run& r, int lane, const uint32_t (&b)[SEGS]) {
    const int k = lane & 3;
    const uint32_t mine = k == 0 ? b[0] : k == 1 ? b[1] : k == 2 ? b[2] : b[3];
    if (k < r.full)
        a.exps[r.row * a.ld_exps + r.c / ISO_ACT_GROUP + k * (TRAIN_SEG / ISO_ACT_GROUP)] = (uint8_t)mine;
}

template <typename T>
__device__ __forceinline__ uint2 encode_raw(const Raw8<T>& x, const float (&v)[8], uint32_t& b) {
    b = act_exp_byte(group_max(x.abs_max()));
    return act_codes(v, b);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_act_pack(const T* x, long long ld, int cols, ActView out, Items it) {
    ACT_FOR_RUNS {
        const Run r(it, i, lane, cols, VEC);
        const T* src = x + r.row * ld + r.c;
        uint8_t* codes = out.codes + r.row * out.ld_codes + r.c;
        Raw8<T> raw[SEGS];
#pragma unroll
        for (int k = 0; k < SEGS; ++k)
            if (VEC && k < r.full) raw[k].load(src + k * TRAIN_SEG);
        uint32_t b[SEGS] = {};
#pragma unroll
        for (int k = 0; k < SEGS; ++k) {
            float v[8];
            if (VEC && k < r.full) {
                raw[k].get(v);
                *reinterpret_cast<uint2*>(codes + k * TRAIN_SEG) = encode_raw(raw[k], v, b[k]);
            } else if (r.c - lane * 8 + k * TRAIN_SEG < cols) {
                const int c = r.c + k * TRAIN_SEG;
                load8<false>(x + r.row * ld, c, cols, v);
                uint2 q;
                const uint32_t e = act_encode(v, q);
                act_store(out, r.row, c, cols, q, e);
            }
        }
        store_exps(out, r, lane, b);
    }
}

template <typename T, bool VEC>
__device__ __forceinline__ void unpack_run(const ActView& in, int cols, T* out, long long ld, const Run& r, int lane) {
    T* dst = out + r.row * ld + r.c;
    const uint8_t* codes = in.codes + r.row * in.ld_codes + r.c;
    const uint8_t* exps = in.exps + r.row * in.ld_exps + r.c / ISO_ACT_GROUP;
    uint2 q[SEGS];
    uint32_t b[SEGS];
#pragma unroll
    for (int k = 0; k < SEGS; ++k)
        if (VEC && k < r.full) {
            q[k] = __ldcs(reinterpret_cast<const uint2*>(codes + k * TRAIN_SEG));
            b[k] = exps[k * (TRAIN_SEG / ISO_ACT_GROUP)];
        }
#pragma unroll
    for (int k = 0; k < SEGS; ++k) {
        float v[8];
        if (VEC && k < r.full) {
            act_decode(q[k], b[k], v);
            put8(dst + k * TRAIN_SEG, v);
        } else if (r.c - lane * 8 + k * TRAIN_SEG < cols) {
            const int c = r.c + k * TRAIN_SEG;
            act_load(in, r.row, c, cols, q[k], b[k]);
            act_decode(q[k], b[k], v);
            store8<VEC>(out + r.row * ld, c, cols, v);
        }
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_act_unpack(ActView in, int cols, T* out, long long ld, Items it) {
    ACT_FOR_RUNS {
        const Run r(it, i, lane, cols, VEC);
        unpack_run<T, VEC>(in, cols, out, ld, r, lane);
    }
}

// The weight gradient's operands.  The first `unpack_blocks` blocks decode x;
// the others write dY as bf16 parts with rows on 16-byte boundaries.  Parts of
// a binary32 value are its leading eight significant bits, cut off (not
// rounded, so that none overflows), then those of the remainder, twice: 24
// bits in all.  A NaN or an infinity stays in the first part.
struct PartsArgs {
    const void* dy;
    long long ldd_in;
    int cols;
    __nv_bfloat16* out;
    long long ldd, part_stride, n;     // n: pieces of eight channels, `segs` a row
    int segs;
};
template <typename T>
__global__ void __launch_bounds__(ACT_TPB) k_wgrad_operands(ActView in, int cols, __nv_bfloat16* x, long long ldx,
                                                            Items it, unsigned unpack_blocks, PartsArgs p) {
    start_next();
    wait_before();
    const int lane = threadIdx.x & 31;
    if (blockIdx.x < unpack_blocks) {
        for (long long i = (long long)blockIdx.x * ACT_WPB + (threadIdx.x >> 5); i < it.n; i += (long long)unpack_blocks * ACT_WPB) {
            const Run r(it, i, lane, cols, true);
            unpack_run<__nv_bfloat16, true>(in, cols, x, ldx, r, lane);
        }
        return;
    }
    const long long threads = (long long)(gridDim.x - unpack_blocks) * ACT_TPB;
    for (long long i = (long long)(blockIdx.x - unpack_blocks) * ACT_TPB + threadIdx.x; i < p.n; i += threads) {
        const long long t = i / p.segs;
        const int c = (int)(i - t * p.segs) * 8;
        float v[8];
        load8<false>(static_cast<const T*>(p.dy) + t * p.ldd_in, c, p.cols, v);
        __nv_bfloat16* o = p.out + t * p.ldd + c;
        if constexpr (sizeof(T) == 2) {
            put8(o, v);
        } else {
#pragma unroll
            for (int q = 0; q < WGRAD_PARTS; ++q) {
                float hi[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t b = __float_as_uint(v[j]);
                    if ((b & 0x7FFFFFFFu) > 0x7F800000u) b |= 0x400000u;     // a NaN stays one without its low bits
                    hi[j] = __uint_as_float(b & 0xFFFF0000u);
                    v[j] = (b & 0x7F800000u) == 0x7F800000u ? 0.0f : v[j] - hi[j];
                }
                put8(o + q * p.part_stride, hi);
            }
        }
    }
}

// s = 1 / (1 + exp(-x)) and 1 - s, both without cancellation and down to the
// subnormals: with e = exp(-|x|) they are 1 / (1 + e) and e / (1 + e), the
// divisor in [1, 2].  bfloat16 outputs take the fast exponential and reciprocal
// (a few binary32 ulps, 1.2 more for every unit of |x|; a bfloat16 ulp is 2^16
// of them), binary32 outputs CUDA's expf and an IEEE division.
template <typename T>
__device__ __forceinline__ void sigmoid(float x, float& s, float& rest) {
    const float e = sizeof(T) == 2 ? __expf(-fabsf(x)) : expf(-fabsf(x));
    const float r = sizeof(T) == 2 ? __fdividef(1.0f, 1.0f + e) : __fdiv_rn(1.0f, 1.0f + e);
    const float er = e * r;
    s = x < 0.0f ? er : r;
    rest = x < 0.0f ? r : er;
}
// x s.  (As x / (1 + exp(-x)) in one fast division it was 0 below x = -87.3,
// where the divisor passes 2^126 and x s is still a normal number.)
template <typename T>
__device__ __forceinline__ float silu(float x) {
    float s, rest;
    sigmoid<T>(x, s, rest);
    return x * s;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(sizeof(T) == 2 ? ACT_TPB : SWIGLU_F32_TPB) k_swiglu_pack(const T* gate, long long ldg, const T* up, long long ldu,
                                                         T* h, long long ldh, int cols, ActView gp, ActView up_p,
                                                         Items it) {
    ACT_FOR_RUNS {
        const Run r(it, i, lane, cols, VEC);
        const T* sg = gate + r.row * ldg + r.c;
        const T* su = up + r.row * ldu + r.c;
        T* dst = h + r.row * ldh + r.c;
        uint8_t* cg = gp.codes + r.row * gp.ld_codes + r.c;
        uint8_t* cu = up_p.codes + r.row * up_p.ld_codes + r.c;
        Raw8<T> rg[SEGS], ru[SEGS];
#pragma unroll
        for (int k = 0; k < SEGS; ++k)
            if (VEC && k < r.full) {
                rg[k].load(sg + k * TRAIN_SEG);
                ru[k].load(su + k * TRAIN_SEG);
            }
        uint32_t bg[SEGS] = {}, bu[SEGS] = {};
#pragma unroll
        for (int k = 0; k < SEGS; ++k) {
            float g[8], u[8], o[8];
            if (VEC && k < r.full) {
                rg[k].get(g);
                ru[k].get(u);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = silu<T>(g[j]) * u[j];
                put8(dst + k * TRAIN_SEG, o);
                *reinterpret_cast<uint2*>(cg + k * TRAIN_SEG) = encode_raw(rg[k], g, bg[k]);
                *reinterpret_cast<uint2*>(cu + k * TRAIN_SEG) = encode_raw(ru[k], u, bu[k]);
            } else if (r.c - lane * 8 + k * TRAIN_SEG < cols) {
                const int c = r.c + k * TRAIN_SEG;
                load8<false>(gate + r.row * ldg, c, cols, g);
                load8<false>(up + r.row * ldu, c, cols, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = silu<T>(g[j]) * u[j];
                store8<false>(h + r.row * ldh, c, cols, o);
                uint2 q;
                uint32_t b = act_encode(g, q);
                act_store(gp, r.row, c, cols, q, b);
                b = act_encode(u, q);
                act_store(up_p, r.row, c, cols, q, b);
            }
        }
        store_exps(gp, r, lane, bg);
        store_exps(up_p, r, lane, bu);
    }
}

template <typename T>
__device__ __forceinline__ void swiglu_grads(const float (&d)[8], const float (&g)[8], const float (&u)[8],
                                             float (&og)[8], float (&ou)[8], float (&oh)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float s, rest;
        sigmoid<T>(g[j], s, rest);
        const float gs = g[j] * s;
        ou[j] = d[j] * gs;
        oh[j] = gs * u[j];
        og[j] = d[j] * u[j] * (s * (1.0f + g[j] * rest));
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_swiglu_grad(const T* dh, long long ldd, ActView gp, ActView up_p,
                                                         int cols, T* d_gate, long long ldg, T* d_up, long long ldu,
                                                         T* h, long long ldh, Items it) {
    ACT_FOR_RUNS {
        const Run r(it, i, lane, cols, VEC);
        const T* sd = dh + r.row * ldd + r.c;
        T* dg = d_gate + r.row * ldg + r.c;
        T* du = d_up + r.row * ldu + r.c;
        T* hh = h + r.row * ldh + r.c;
        const uint8_t* cg = gp.codes + r.row * gp.ld_codes + r.c;
        const uint8_t* cu = up_p.codes + r.row * up_p.ld_codes + r.c;
        const uint8_t* eg = gp.exps + r.row * gp.ld_exps + r.c / ISO_ACT_GROUP;
        const uint8_t* eu = up_p.exps + r.row * up_p.ld_exps + r.c / ISO_ACT_GROUP;
        Raw8<T> rd[SEGS];
        uint2 qg[SEGS], qu[SEGS];
        uint32_t bg[SEGS], bu[SEGS];
#pragma unroll
        for (int k = 0; k < SEGS; ++k)
            if (VEC && k < r.full) {
                rd[k].load(sd + k * TRAIN_SEG);
                qg[k] = __ldcs(reinterpret_cast<const uint2*>(cg + k * TRAIN_SEG));
                qu[k] = __ldcs(reinterpret_cast<const uint2*>(cu + k * TRAIN_SEG));
                bg[k] = eg[k * (TRAIN_SEG / ISO_ACT_GROUP)];
                bu[k] = eu[k * (TRAIN_SEG / ISO_ACT_GROUP)];
            }
#pragma unroll
        for (int k = 0; k < SEGS; ++k) {
            float d[8], g[8], u[8], og[8], ou[8], oh[8];
            if (VEC && k < r.full) {
                rd[k].get(d);
                act_decode(qg[k], bg[k], g);
                act_decode(qu[k], bu[k], u);
                swiglu_grads<T>(d, g, u, og, ou, oh);
                put8(dg + k * TRAIN_SEG, og);
                put8(du + k * TRAIN_SEG, ou);
                if (h) put8(hh + k * TRAIN_SEG, oh);
            } else if (r.c - lane * 8 + k * TRAIN_SEG < cols) {
                const int c = r.c + k * TRAIN_SEG;
                act_load(gp, r.row, c, cols, qg[k], bg[k]);
                act_load(up_p, r.row, c, cols, qu[k], bu[k]);
                load8<false>(dh + r.row * ldd, c, cols, d);
                act_decode(qg[k], bg[k], g);
                act_decode(qu[k], bu[k], u);
                swiglu_grads<T>(d, g, u, og, ou, oh);
                store8<false>(d_gate + r.row * ldg, c, cols, og);
                store8<false>(d_up + r.row * ldu, c, cols, ou);
                if (h) store8<false>(h + r.row * ldh, c, cols, oh);
            }
        }
    }
}

ActView view(const iso_act* a) {
    return {static_cast<uint8_t*>(a->codes), static_cast<uint8_t*>(a->exps), (long long)a->ld_codes,
            (long long)a->ld_exps};
}
Items items_of(int64_t rows, int64_t cols) {
    const int runs = (int)((cols + SEGS * TRAIN_SEG - 1) / (SEGS * TRAIN_SEG));
    return {(long long)rows * runs, runs};
}
unsigned act_grid(const Items& it, int tpb = ACT_TPB) {
    return (unsigned)std::min((it.n + tpb / 32 - 1) / (tpb / 32), (long long)EXTENT_LIMIT);
}

}  // namespace

int launch_wgrad_operands(const iso_act* pack, __nv_bfloat16* x, long long ldx, const iso_mat* dy,
                          __nv_bfloat16* parts, long long ldd, cudaStream_t s) {
    const Items it = items_of(pack->rows, pack->cols);
    const unsigned unpack_blocks = std::min(act_grid(it), 1u << 30);
    PartsArgs p{};
    unsigned part_blocks = 0;
    if (dy) {
        const int segs = (int)((dy->cols + 7) / 8);
        p = {dy->data, (long long)dy->ld, (int)dy->cols, parts, ldd, (long long)dy->rows * ldd, (long long)dy->rows * segs, segs};
        part_blocks = (unsigned)std::min((p.n + ACT_TPB - 1) / ACT_TPB, 1LL << 30);
    }
    if (dy && dy->dtype == ISO_F32)
        TRAIN_LAUNCH(launch_early(k_wgrad_operands<float>, unpack_blocks + part_blocks, ACT_TPB, 0, s, view(pack),
                                  (int)pack->cols, x, ldx, it, unpack_blocks, p));
    else
        TRAIN_LAUNCH(launch_early(k_wgrad_operands<__nv_bfloat16>, unpack_blocks + part_blocks, ACT_TPB, 0, s, view(pack),
                                  (int)pack->cols, x, ldx, it, unpack_blocks, p));
    return ISO_OK;
}

namespace {

template <typename F>
int dispatch_act(int32_t dtype, bool vec, F&& f) {
    if (dtype == ISO_BF16) {
        using T = __nv_bfloat16;
        return vec ? f((T*)nullptr, std::true_type{}) : f((T*)nullptr, std::false_type{});
    }
    return vec ? f((float*)nullptr, std::true_type{}) : f((float*)nullptr, std::false_type{});
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_act_pack(const iso_mat* x, const iso_act* pack, void* stream) {
    ISO_TRY(check_mat(x));
    ISO_TRY(check_act(pack));
    if (x->rows != pack->rows || x->cols != pack->cols) return ISO_ERR_SHAPE;
    if (share_bytes(bytes_of(x), codes_of(pack)) || share_bytes(bytes_of(x), exps_of(pack)) ||
        share_bytes(codes_of(pack), exps_of(pack)))
        return ISO_ERR_ARG;
    if (x->rows == 0 || x->cols == 0) return ISO_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Items it = items_of(x->rows, x->cols);
    return dispatch_act(x->dtype, rows_aligned(x), [&](auto* tp, auto vec) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        TRAIN_LAUNCH((k_act_pack<T, decltype(vec)::value><<<act_grid(it), ACT_TPB, 0, s>>>(
            static_cast<const T*>(x->data), x->ld, (int)x->cols, view(pack), it)));
        return ISO_OK;
    });
}

int32_t iso_act_unpack(const iso_act* pack, const iso_mat* out, void* stream) {
    ISO_TRY(check_mat(out));
    ISO_TRY(check_act(pack));
    if (out->rows != pack->rows || out->cols != pack->cols) return ISO_ERR_SHAPE;
    if (share_bytes(bytes_of(out), codes_of(pack)) || share_bytes(bytes_of(out), exps_of(pack))) return ISO_ERR_ARG;
    if (out->rows == 0 || out->cols == 0) return ISO_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Items it = items_of(out->rows, out->cols);
    return dispatch_act(out->dtype, rows_aligned(out), [&](auto* tp, auto vec) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        TRAIN_LAUNCH((k_act_unpack<T, decltype(vec)::value><<<act_grid(it), ACT_TPB, 0, s>>>(
            view(pack), (int)out->cols, static_cast<T*>(out->data), out->ld, it)));
        return ISO_OK;
    });
}

int32_t iso_swiglu_pack(const iso_mat* gate, const iso_mat* up, const iso_mat* h, const iso_act* gate_pack,
                        const iso_act* up_pack, void* stream) {
    const iso_mat* mats[3] = {gate, up, h};
    const iso_act* acts[2] = {gate_pack, up_pack};
    for (const iso_mat* m : mats) {
        ISO_TRY(check_mat(m));
        if (m->rows != gate->rows || m->cols != gate->cols) return ISO_ERR_SHAPE;
        if (m->dtype != gate->dtype) return ISO_ERR_DTYPE;
    }
    Bytes2D outs[5] = {bytes_of(h)};
    int n_outs = 1;
    for (const iso_act* a : acts) {
        ISO_TRY(check_act(a));
        if (a->rows != gate->rows || a->cols != gate->cols) return ISO_ERR_SHAPE;
        outs[n_outs++] = codes_of(a);
        outs[n_outs++] = exps_of(a);
    }
    for (int i = 0; i < n_outs; ++i) {
        if (share_bytes(outs[i], bytes_of(gate)) || share_bytes(outs[i], bytes_of(up))) return ISO_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (share_bytes(outs[i], outs[j])) return ISO_ERR_ARG;
    }
    if (gate->rows == 0 || gate->cols == 0) return ISO_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Items it = items_of(gate->rows, gate->cols);
    const bool vec = rows_aligned(gate) && rows_aligned(up) && rows_aligned(h);
    return dispatch_act(gate->dtype, vec, [&](auto* tp, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        constexpr int tpb = sizeof(T) == 2 ? ACT_TPB : SWIGLU_F32_TPB;
        TRAIN_LAUNCH((k_swiglu_pack<T, decltype(v)::value><<<act_grid(it, tpb), tpb, 0, s>>>(
            static_cast<const T*>(gate->data), gate->ld, static_cast<const T*>(up->data), up->ld,
            static_cast<T*>(h->data), h->ld, (int)gate->cols, view(gate_pack), view(up_pack), it)));
        return ISO_OK;
    });
}

int32_t iso_swiglu_grad(const iso_mat* dh, const iso_act* gate_pack, const iso_act* up_pack, const iso_mat* d_gate,
                        const iso_mat* d_up, const iso_mat* h, void* stream) {
    const iso_mat* mats[4] = {dh, d_gate, d_up, h};
    Bytes2D outs[3];
    int n_outs = 0;
    for (int i = 0; i < 4; ++i) {
        const iso_mat* m = mats[i];
        if (i == 3 && !m) break;
        ISO_TRY(check_mat(m));
        if (m->rows != dh->rows || m->cols != dh->cols) return ISO_ERR_SHAPE;
        if (m->dtype != dh->dtype) return ISO_ERR_DTYPE;
        if (i) outs[n_outs++] = bytes_of(m);
    }
    for (const iso_act* a : {gate_pack, up_pack}) {
        ISO_TRY(check_act(a));
        if (a->rows != dh->rows || a->cols != dh->cols) return ISO_ERR_SHAPE;
    }
    for (int i = 0; i < n_outs; ++i) {
        if (share_bytes(outs[i], bytes_of(dh))) return ISO_ERR_ARG;
        for (const iso_act* a : {gate_pack, up_pack})
            if (share_bytes(outs[i], codes_of(a)) || share_bytes(outs[i], exps_of(a))) return ISO_ERR_ARG;
        for (int j = 0; j < i; ++j)
            if (share_bytes(outs[i], outs[j])) return ISO_ERR_ARG;
    }
    if (dh->rows == 0 || dh->cols == 0) return ISO_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Items it = items_of(dh->rows, dh->cols);
    const bool vec = rows_aligned(dh) && rows_aligned(d_gate) && rows_aligned(d_up) && (!h || rows_aligned(h));
    return dispatch_act(dh->dtype, vec, [&](auto* tp, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        TRAIN_LAUNCH((k_swiglu_grad<T, decltype(v)::value><<<act_grid(it), ACT_TPB, 0, s>>>(
            static_cast<const T*>(dh->data), dh->ld, view(gate_pack), view(up_pack), (int)dh->cols,
            static_cast<T*>(d_gate->data), d_gate->ld, static_cast<T*>(d_up->data), d_up->ld,
            h ? static_cast<T*>(h->data) : nullptr, h ? h->ld : 0, it)));
        return ISO_OK;
    });
}

}  // extern "C"
