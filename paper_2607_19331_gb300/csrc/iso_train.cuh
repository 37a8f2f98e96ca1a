// iso_train.cuh -- helpers shared by the training-step operators: argument
// checks of strided matrices and checkpoints (host), 8-element row accesses
// and the checkpoint's number format (device).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "iso.h"
#include "iso_gemm.cuh"

namespace iso {

constexpr int TRAIN_SEG = 256;   // channels of one row that a warp takes at a time (8 per lane)

#define TRAIN_LAUNCH(...) do { const int _slot = prof_begin(3, s); __VA_ARGS__; prof_end(_slot, s); \
                               if (cudaGetLastError() != cudaSuccess) return ISO_ERR_CUDA; } while (0)

// ---------------------------------------------------------------------------
// host: argument checks
// ---------------------------------------------------------------------------
inline int elem_size(int32_t dtype) { return dtype == ISO_BF16 ? 2 : 4; }
inline int64_t act_cols_padded(int64_t cols) { return (cols + ISO_ACT_GROUP - 1) / ISO_ACT_GROUP * ISO_ACT_GROUP; }
inline int64_t act_exps_padded(int64_t cols) {
    return ((cols + ISO_ACT_GROUP - 1) / ISO_ACT_GROUP + 7) / 8 * 8;
}

constexpr int64_t EXTENT_LIMIT = 0x7FFF0000LL;    // below 2^31 with room for a kernel's last step
constexpr int64_t STRIDE_LIMIT = 1LL << 36;
constexpr int64_t SPAN_LIMIT = 1LL << 52;         // rows x stride
inline bool span_too_large(int64_t rows, int64_t ld) { return rows > 1 && ld > SPAN_LIMIT / rows; }

inline int check_mat(const iso_mat* m) {
    if (!m || m->reserved != 0) return ISO_ERR_ARG;
    if (m->rows < 0 || m->cols < 0 || m->ld < m->cols) return ISO_ERR_SHAPE;
    if (m->rows > EXTENT_LIMIT || m->cols > EXTENT_LIMIT || m->ld > STRIDE_LIMIT || span_too_large(m->rows, m->ld))
        return ISO_ERR_UNSUPPORTED;
    if (m->dtype != ISO_BF16 && m->dtype != ISO_F32) return ISO_ERR_DTYPE;
    if (m->rows == 0 || m->cols == 0) return ISO_OK;
    if (!m->data) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(m->data) % elem_size(m->dtype)) return ISO_ERR_ALIGN;
    return ISO_OK;
}

inline int check_act(const iso_act* a) {
    if (!a) return ISO_ERR_ARG;
    if (a->rows < 0 || a->cols < 0) return ISO_ERR_SHAPE;
    if (a->rows > EXTENT_LIMIT || a->cols > EXTENT_LIMIT || a->ld_codes > STRIDE_LIMIT || a->ld_exps > STRIDE_LIMIT ||
        span_too_large(a->rows, a->ld_codes) || span_too_large(a->rows, a->ld_exps))
        return ISO_ERR_UNSUPPORTED;
    if (a->ld_codes < act_cols_padded(a->cols) || a->ld_exps < act_exps_padded(a->cols)) return ISO_ERR_SHAPE;
    if (a->ld_codes % ISO_ACT_GROUP || a->ld_exps % 8) return ISO_ERR_ALIGN;
    if (a->rows == 0 || a->cols == 0) return ISO_OK;
    if (!a->codes || !a->exps) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(a->codes) & 15u || reinterpret_cast<uintptr_t>(a->exps) & 7u) return ISO_ERR_ALIGN;
    return ISO_OK;
}

// A rectangle of bytes: `rows` runs of `width` bytes, `stride` apart.
struct Bytes2D {
    uintptr_t at;
    uint64_t rows, width, stride;
};
inline Bytes2D bytes_of(const iso_mat* m) {
    const uint64_t e = elem_size(m->dtype);
    return {reinterpret_cast<uintptr_t>(m->data), (uint64_t)m->rows, (uint64_t)m->cols * e, (uint64_t)m->ld * e};
}
inline Bytes2D codes_of(const iso_act* a) {
    return {reinterpret_cast<uintptr_t>(a->codes), (uint64_t)a->rows, (uint64_t)act_cols_padded(a->cols),
            (uint64_t)a->ld_codes};
}
inline Bytes2D exps_of(const iso_act* a) {
    return {reinterpret_cast<uintptr_t>(a->exps), (uint64_t)a->rows, (uint64_t)act_exps_padded(a->cols),
            (uint64_t)a->ld_exps};
}
// Whether two rectangles share a byte.  Exact for equal strides (columns of
// one buffer); otherwise whether their address ranges meet.
inline bool share_bytes(const Bytes2D& a, const Bytes2D& b) {
    if (!a.rows || !a.width || !b.rows || !b.width) return false;
    const uintptr_t ea = a.at + (a.rows - 1) * a.stride + a.width, eb = b.at + (b.rows - 1) * b.stride + b.width;
    if (ea <= b.at || eb <= a.at) return false;
    if (a.stride != b.stride || a.rows == 1 || b.rows == 1) {
        // a single row may lie in the gaps of the other rectangle
        const Bytes2D& one = a.rows == 1 ? a : b;
        const Bytes2D& many = a.rows == 1 ? b : a;
        if (one.rows != 1) return true;
        if (many.rows == 1) return true;                        // the ranges meet
        if (one.at < many.at) return true;                      // reaches into the first row
        const uint64_t off = (one.at - many.at) % many.stride;
        const bool last = (one.at - many.at) / many.stride >= many.rows - 1;
        return off < many.width || (!last && off + one.width > many.stride);
    }
    const Bytes2D& lo = a.at <= b.at ? a : b;
    const Bytes2D& hi = a.at <= b.at ? b : a;
    const uint64_t row = (hi.at - lo.at) / lo.stride, off = (hi.at - lo.at) % lo.stride;
    // hi's first row starts in lo's row `row` at `off`, and may run into the next
    return off < lo.width || (off + hi.width > lo.stride && row + 1 < lo.rows);
}

// rows start on 16-byte boundaries
inline bool rows_aligned(const iso_mat* m) {
    return m->rows == 0 || m->cols == 0 ||
           ((reinterpret_cast<uintptr_t>(m->data) & 15u) == 0 && (m->rows == 1 || (m->ld * elem_size(m->dtype)) % 16 == 0));
}

// The clock of a bounded wait: look() at the time now (ns) says whether the wait
// has lasted longer than its limit.  The GPU's timer runs on while another
// process has the GPU, so the time between two looks counts WAIT_GAP_NS at most:
// a kernel that was away does not give up when it comes back.  (Looks are
// microseconds apart; 2 s take a hundred of the longest gaps.)
constexpr uint64_t WAIT_GAP_NS = 20000000;
struct WaitClock {
    uint64_t last = 0, waited = 0;
    __host__ __device__ __forceinline__ bool look(uint64_t now, uint64_t limit_ns) {
        if (last) waited += now - last < WAIT_GAP_NS ? now - last : WAIT_GAP_NS;
        last = now;
        return waited > limit_ns;
    }
};

// SMs of the current device (queried once per device)
int train_sms();

// A kernel that may be launched while the one before it on the stream still
// runs; it calls wait_before (below) ahead of its first access to memory.  The
// one before lets it start early by calling start_next, which says nothing
// about its own work being done.
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// The weight gradient's bf16 operands, in one kernel (iso_act.cu): x (rows of
// ldx) <- the values of pack; with dy, parts (WGRAD_PARTS or 1 matrices of
// rows x ldd) <- dY.  ldx and ldd are multiples of 8.
constexpr int WGRAD_PARTS = 3;
int launch_wgrad_operands(const iso_act* pack, __nv_bfloat16* x, long long ldx, const iso_mat* dy,
                          __nv_bfloat16* parts, long long ldd, cudaStream_t s);

// ---------------------------------------------------------------------------
// device: rows, eight elements at a time
// ---------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f32(float v, float& o) { o = v; }
__device__ __forceinline__ void from_f32(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }

__device__ __forceinline__ void bf16x2_to_f32(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t f32_to_bf16x2(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&v);
}

// v[i] = row[c + i] for c + i < cols, else 0.  VEC: the row starts on a
// 16-byte boundary and c is a multiple of 8.
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int c, int cols, float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4*>(row + c));
        bf16x2_to_f32(w.x, v[0], v[1]);
        bf16x2_to_f32(w.y, v[2], v[3]);
        bf16x2_to_f32(w.z, v[4], v[5]);
        bf16x2_to_f32(w.w, v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? __bfloat162float(row[c + i]) : 0.0f;
    }
}
template <bool VEC>
__device__ __forceinline__ void load8(const float* row, int c, int cols, float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(row + c));
        const float4 b = __ldcs(reinterpret_cast<const float4*>(row + c + 4));
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? row[c + i] : 0.0f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* row, int c, int cols, const float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        uint4 w;
        w.x = f32_to_bf16x2(v[0], v[1]);
        w.y = f32_to_bf16x2(v[2], v[3]);
        w.z = f32_to_bf16x2(v[4], v[5]);
        w.w = f32_to_bf16x2(v[6], v[7]);
        *reinterpret_cast<uint4*>(row + c) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = __float2bfloat16_rn(v[i]);
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* row, int c, int cols, const float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = v[i];
    }
}

// ---------------------------------------------------------------------------
// device: the checkpoint's number format (iso_act)
// ---------------------------------------------------------------------------
// Exponent byte of a group whose largest magnitude has the binary32 bits
// `amax`.  With amax = 1.f 2^(E - 127), amax <= 127 2^e = 1.984375 2^(e + 6)
// holds for e = E - 133 when 1.f <= 1.984375 (mantissa bits <= 0x7E0000) and
// for e = E - 132 otherwise, where adding 0x1FFFF carries into the exponent;
// the byte is e + 127, at least 1 (e = -126).
__device__ __forceinline__ uint32_t act_exp_byte(uint32_t amax) {
    const int b = (int)((amax + 0x1FFFFu) >> 23) - 6;
    return amax >= 0x7F800000u ? 255u : (uint32_t)max(b, 1);   // 255: a NaN or an infinity in the group
}
// 2^(b - 127) for b in 1 .. 254, +Inf for 255 (its codes are 0: 0 * Inf = NaN)
__device__ __forceinline__ float act_scale(uint32_t b) { return __uint_as_float(b << 23); }

// largest magnitude of eight values, as binary32 bits; any NaN counts as one
__device__ __forceinline__ uint32_t abs_max8(const float (&v)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return a;
}
// the four lanes of a group; every lane of the warp calls it
__device__ __forceinline__ uint32_t group_max(uint32_t a) {
    a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    return max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
}
// the low bytes of four words, the first one lowest
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// Codes of eight values under the exponent byte b.  x 2^(127 - b) is exact, so
// adding 1.5 2^23 to it rounds it once, to the nearest integer with halves to
// even, and leaves that integer in the sum's low byte.
__device__ __forceinline__ uint2 act_codes(const float (&v)[8], uint32_t b) {
    const float inv = __uint_as_float((254u - b) << 23);
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(__fmaf_rn(v[i], inv, 12582912.0f));
    if (b >= 249u) {   // 64 * 2^122 is no binary32 number; NaN and Inf groups hold zeros
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = b == 255u ? 0u : (uint32_t)min(max((int)(int8_t)q[i], -63), 63);
    }
    return make_uint2(low_bytes(q[0], q[1], q[2], q[3]), low_bytes(q[4], q[5], q[6], q[7]));
}
// Codes of this lane's eight values, of a group of four lanes; returns the
// exponent byte.  Every lane of the warp calls it.
__device__ __forceinline__ uint32_t act_encode(const float (&v)[8], uint2& codes) {
    const uint32_t b = act_exp_byte(group_max(abs_max8(v)));
    codes = act_codes(v, b);
    return b;
}
// Eight values.  A code's byte with its top bit flipped, under the exponent of
// 2^23, is 2^23 + 128 + code: taking the offset off and scaling are both exact
// (b = 255: 0 * Inf = NaN).
__device__ __forceinline__ void act_decode(uint2 codes, uint32_t b, float (&v)[8]) {
    const float s = act_scale(b);
    const uint32_t x = codes.x ^ 0x80808080u, y = codes.y ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (__uint_as_float(__byte_perm(x, 0x4B000000u, 0x7440u + i)) - 8388736.0f) * s;
        v[4 + i] = (__uint_as_float(__byte_perm(y, 0x4B000000u, 0x7440u + i)) - 8388736.0f) * s;
    }
}

// eight entries of a row that starts on a 16-byte boundary, as loaded
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load_shared(const void* p) { w = *static_cast<const uint4*>(p); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        bf16x2_to_f32(w.x, v[0], v[1]);
        bf16x2_to_f32(w.y, v[2], v[3]);
        bf16x2_to_f32(w.z, v[4], v[5]);
        bf16x2_to_f32(w.w, v[6], v[7]);
    }
    // magnitudes compared two by two: as for binary32, their bits order them, NaN above all
    __device__ __forceinline__ uint32_t abs_max() const {
        const uint32_t m = 0x7FFF7FFFu;
        const uint32_t a = __vmaxu2(__vmaxu2(w.x & m, w.y & m), __vmaxu2(w.z & m, w.w & m));
        return max(a & 0xFFFF0000u, a << 16);
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load_shared(const void* p) {
        a = static_cast<const float4*>(p)[0];
        b = static_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void load(const float* p) {
        a = __ldcs(reinterpret_cast<const float4*>(p));
        b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ uint32_t abs_max() const {
        float v[8];
        get(v);
        return abs_max8(v);
    }
};

__device__ __forceinline__ void put8(__nv_bfloat16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3]),
                                              f32_to_bf16x2(v[4], v[5]), f32_to_bf16x2(v[6], v[7]));
}
// 32 bytes in one store where they are aligned to that: two 16-byte ones write
// half sectors
__device__ __forceinline__ void put8(float* p, const float (&v)[8]) {
    if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     :: "l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
    } else {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

}  // namespace iso
