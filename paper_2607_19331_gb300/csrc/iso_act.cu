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

namespace iso {

int train_sms() {
    static int sms[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
    if (!sms[dev]) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 152;
        sms[dev] = n;
    }
    return sms[dev];
}

namespace {

constexpr int ACT_TPB = 256;
constexpr int ACT_WPB = ACT_TPB / 32;

struct ActView {
    uint8_t* codes;
    uint8_t* exps;
    long long ld_codes, ld_exps;
};

// Segments of a rows x cols matrix, row after row: item i is segment i % segs
// of row i / segs.
struct Items {
    long long n;
    int segs;
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

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_act_pack(const T* x, long long ld, int cols, ActView out, Items it) {
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * ACT_WPB;
    for (long long i = (long long)blockIdx.x * ACT_WPB + (threadIdx.x >> 5); i < it.n; i += warps) {
        const long long row = i / it.segs;
        const int c = (int)(i - row * it.segs) * TRAIN_SEG + lane * 8;
        float v[8];
        load8<VEC>(x + row * ld, c, cols, v);
        uint2 q;
        const uint32_t b = act_encode(v, q);
        act_store(out, row, c, cols, q, b);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_act_unpack(ActView in, int cols, T* out, long long ld, Items it) {
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * ACT_WPB;
    for (long long i = (long long)blockIdx.x * ACT_WPB + (threadIdx.x >> 5); i < it.n; i += warps) {
        const long long row = i / it.segs;
        const int c = (int)(i - row * it.segs) * TRAIN_SEG + lane * 8;
        uint2 q;
        uint32_t b;
        act_load(in, row, c, cols, q, b);
        float v[8];
        act_decode(q, b, v);
        store8<VEC>(out + row * ld, c, cols, v);
    }
}

// s = 1 / (1 + exp(-x)) and 1 - s, both without cancellation and down to the
// subnormals: with e = exp(-|x|) they are 1 / (1 + e) and e / (1 + e).
__device__ __forceinline__ void sigmoid(float x, float& s, float& rest) {
    const float e = expf(-fabsf(x)), r = __fdiv_rn(1.0f, 1.0f + e), er = e * r;
    s = x < 0.0f ? er : r;
    rest = x < 0.0f ? r : er;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_swiglu_pack(const T* gate, long long ldg, const T* up, long long ldu,
                                                         T* h, long long ldh, int cols, ActView gp, ActView up_p,
                                                         Items it) {
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * ACT_WPB;
    for (long long i = (long long)blockIdx.x * ACT_WPB + (threadIdx.x >> 5); i < it.n; i += warps) {
        const long long row = i / it.segs;
        const int c = (int)(i - row * it.segs) * TRAIN_SEG + lane * 8;
        float g[8], u[8], o[8];
        load8<VEC>(gate + row * ldg, c, cols, g);
        load8<VEC>(up + row * ldu, c, cols, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float s, rest;
            sigmoid(g[j], s, rest);
            o[j] = g[j] * s * u[j];
        }
        store8<VEC>(h + row * ldh, c, cols, o);
        uint2 q;
        uint32_t b = act_encode(g, q);
        act_store(gp, row, c, cols, q, b);
        b = act_encode(u, q);
        act_store(up_p, row, c, cols, q, b);
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ACT_TPB) k_swiglu_grad(const T* dh, long long ldd, ActView gp, ActView up_p,
                                                         int cols, T* d_gate, long long ldg, T* d_up, long long ldu,
                                                         T* h, long long ldh, Items it) {
    const int lane = threadIdx.x & 31;
    const long long warps = (long long)gridDim.x * ACT_WPB;
    for (long long i = (long long)blockIdx.x * ACT_WPB + (threadIdx.x >> 5); i < it.n; i += warps) {
        const long long row = i / it.segs;
        const int c = (int)(i - row * it.segs) * TRAIN_SEG + lane * 8;
        uint2 qg, qu;
        uint32_t bg, bu;
        float d[8], g[8], u[8], og[8], ou[8], oh[8];
        act_load(gp, row, c, cols, qg, bg);
        act_load(up_p, row, c, cols, qu, bu);
        load8<VEC>(dh + row * ldd, c, cols, d);
        act_decode(qg, bg, g);
        act_decode(qu, bu, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float s, rest;
            sigmoid(g[j], s, rest);
            const float gs = g[j] * s;
            ou[j] = d[j] * gs;
            oh[j] = gs * u[j];
            og[j] = d[j] * u[j] * (s * (1.0f + g[j] * rest));
        }
        store8<VEC>(d_gate + row * ldg, c, cols, og);
        store8<VEC>(d_up + row * ldu, c, cols, ou);
        if (h) store8<VEC>(h + row * ldh, c, cols, oh);
    }
}

ActView view(const iso_act* a) {
    return {static_cast<uint8_t*>(a->codes), static_cast<uint8_t*>(a->exps), (long long)a->ld_codes,
            (long long)a->ld_exps};
}
Items items_of(int64_t rows, int64_t cols) {
    const int segs = (int)((cols + TRAIN_SEG - 1) / TRAIN_SEG);
    return {(long long)rows * segs, segs};
}
int act_grid(const Items& it) {
    return (int)std::max(1LL, std::min((it.n + ACT_WPB - 1) / ACT_WPB, (long long)train_sms() * 8));
}

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
        TRAIN_LAUNCH((k_swiglu_pack<T, decltype(v)::value><<<act_grid(it), ACT_TPB, 0, s>>>(
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
