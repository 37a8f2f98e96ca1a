// iso_distill.cu -- distillation from a teacher's top logits: loss, log-sum-exp
// and the gradient of the logits.
//
// The logits are all of the traffic (K ids and teacher logits a row against a
// vocabulary), and a row takes one exponential an entry for the sum and one for
// the gradient: bound by HBM.  Loss and gradient in one call therefore read the
// logits once:
//   k_distill       a cluster of 1 ... 8 CTAs holds a whole row in registers, as
//                   it was loaded (up to ten 16-byte words a thread), so every
//                   load of a row is in flight at once; statistics per thread,
//                   then warp, CTA and cluster (distributed shared memory), and
//                   the gradient from the same registers.  The K entries are
//                   gathered beside the row and put right after it, by the CTA
//                   that owns their columns.
//   k_distill_long  rows that do not fit, or whose logits and gradient do not
//                   sit alike in 16-byte words: one CTA a row, two passes.
// A row off a 16-byte boundary is taken as its words from the first boundary on;
// the entries before and behind them (under one word each) go one by one.
// Statistics: each thread keeps its maximum m and sum of exp(x - m); pairs are
// joined as (max, s1 exp(m1 - max) + s2 exp(m2 - max)) in a fixed order.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <cmath>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace iso {
namespace {

constexpr int DI_MAX_CLUSTER = 8;
constexpr int DI_MAX_WORDS = 10;         // 16-byte words of a row a thread holds
constexpr float LOG2E = 1.4426950408889634f;

struct DistillArgs {
    const void* z;
    const void* ids;
    const void* teacher;
    void* grad;                          // NULL: loss alone
    const float* dloss;
    const float* lse_in;                 // the gradient alone, from these
    float* loss;
    float* lse;
    int32_t* status;
    long long ldz, ldt, ldg;
    int32_t rows, vocab, top;
    int32_t ids_i64, teacher_f32;
    float tau, inv_tau;
};

// m = -Inf where nothing was seen (then s = 0)
struct Stat {
    float m, s;
};
// exp(x / tau) for a bf16 row by the hardware's exponential (2 ulp, far below the
// rounding of the gradient, and random beside one another in the sum), for a
// binary32 row by expf
template <bool FAST>
struct Exp {
    float c;
    __device__ __forceinline__ explicit Exp(float inv_tau) : c(FAST ? inv_tau * LOG2E : inv_tau) {}
    __device__ __forceinline__ float of(float x) const {
        if constexpr (FAST) {
            float y;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
            return y;
        } else {
            return expf(x);
        }
    }
    __device__ __forceinline__ float below(float x, float top) const { return of((x - top) * c); }   // exp((x - top) / tau)
    // exp(x / tau - m), m given as level(m)
    __device__ __forceinline__ float level(float m) const { return FAST ? m * LOG2E : m; }
    __device__ __forceinline__ float against(float x, float l) const { return of(fmaf(x, c, -l)); }
};
__device__ __forceinline__ Stat join(Stat a, Stat b) {
    const float m = fmaxf(a.m, b.m);
    // equal maxima (two infinities of one sign among them) need no scaling
    const float sa = a.m == m ? a.s : a.s * expf(a.m - m), sb = b.m == m ? b.s : b.s * expf(b.m - m);
    return {m, sa + sb};
}
__device__ __forceinline__ Stat warp_join(Stat a) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const Stat b = {__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o)};
        a = join(a, b);
    }
    return a;
}

__device__ __forceinline__ long long id_at(const DistillArgs& g, long long i) {
    return g.ids_i64 ? static_cast<const long long*>(g.ids)[i] : (long long)static_cast<const int*>(g.ids)[i];
}

// The teacher's side of a row, in shared memory of each CTA: ids (-1: unused),
// probabilities, and the logits at the ids.
struct Top {
    int* id;
    float* p;
    float* z;
};

// NT threads; t.z must be gathered by the caller.  Returns false where the row
// has no used slot with a finite weight (loss and gradient 0).
template <int NT>
__device__ __forceinline__ bool teacher_side(const DistillArgs& g, int row, const Top& t, float* red) {
    float m = -INFINITY;
    bool nan = false;
    for (int k = threadIdx.x; k < g.top; k += NT) {
        const long long v = id_at(g, (long long)row * g.top + k);
        const long long at = (long long)row * g.ldt + k;
        const bool used = v >= 0 && v < g.vocab;
        if (!used && v != -1 && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_INDEX);
        float x = -INFINITY;
        if (used)
            x = (g.teacher_f32 ? static_cast<const float*>(g.teacher)[at]
                               : __bfloat162float(static_cast<const __nv_bfloat16*>(g.teacher)[at])) * g.inv_tau;
        t.id[k] = used ? (int)v : -1;
        t.p[k] = x;
        m = fmaxf(m, x);
        nan |= x != x;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    nan = __any_sync(0xFFFFFFFFu, nan);
    if (lane == 0) red[warp] = nan ? __int_as_float(0x7FFFFFFF) : m;
    __syncthreads();
    m = -INFINITY;
    nan = false;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const float x = red[w];
        m = fmaxf(m, x);
        nan |= x != x;
    }
    if (m == -INFINITY && !nan) return false;
    if (nan) m = __int_as_float(0x7FFFFFFF);
    float s = 0.0f;
    for (int k = threadIdx.x; k < g.top; k += NT) {
        const float x = t.id[k] < 0 ? 0.0f : expf(t.p[k] - m);
        t.p[k] = x;
        s += x;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    __syncthreads();
    if (lane == 0) red[warp] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) s += red[w];
    for (int k = threadIdx.x; k < g.top; k += NT) t.p[k] = t.p[k] / s;
    return true;
}

// sum_k p_k (log p_k - z_k / tau + lse), by the whole CTA, in a fixed order
template <int NT>
__device__ __forceinline__ float divergence(const DistillArgs& g, const Top& t, float lse, float* red) {
    float s = 0.0f;
    for (int k = threadIdx.x; k < g.top; k += NT) {
        const float p = t.p[k];
        if (t.id[k] >= 0 && p != 0.0f) s += p * (logf(p) - (t.z[k] * g.inv_tau - lse));
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    __syncthreads();
    if (lane == 0) red[warp] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) s += red[w];
    return s;
}

// The entries at the teacher's ids among columns [c0, c1): the probabilities of
// all slots with the id, in slot order, off the student's.  Slots of one id write
// the same value.  q(z) is the student's probability.
template <int NT, typename T, typename Q>
__device__ __forceinline__ void put_right(const DistillArgs& g, const Top& t, T* grad, int c0, int c1, float scale, Q q) {
    for (int k = threadIdx.x; k < g.top; k += NT) {
        const int id = t.id[k];
        if (id < c0 || id >= c1) continue;
        float p = 0.0f;
        for (int j = 0; j < g.top; ++j) p += t.id[j] == id ? t.p[j] : 0.0f;
        from_f32(scale * (q(t.z[k]) - p), grad[id]);
    }
}

template <typename T>
struct Word {                            // 16 bytes of a row
    static constexpr int N = 16 / sizeof(T);
    uint4 w;
    __device__ __forceinline__ void get(float (&v)[N]) const {
        if constexpr (sizeof(T) == 2) {
            bf16x2_to_f32(w.x, v[0], v[1]);
            bf16x2_to_f32(w.y, v[2], v[3]);
            bf16x2_to_f32(w.z, v[4], v[5]);
            bf16x2_to_f32(w.w, v[6], v[7]);
        } else {
            v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y);
            v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[N]) {
        if constexpr (sizeof(T) == 2)
            w = make_uint4(f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3]), f32_to_bf16x2(v[4], v[5]),
                           f32_to_bf16x2(v[6], v[7]));
        else
            w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};

// Entries before a row's first 16-byte boundary (all of them for a shorter row)
template <typename T>
__device__ __forceinline__ int entries_before(const T* row, int n) {
    const int off = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / (int)sizeof(T);
    return min(off, n);
}

// m and s of a thread's entries so far, with one more value
__device__ __forceinline__ void add_one(Stat& a, float x) {
    const float m = fmaxf(a.m, x);
    if (m == -INFINITY) {
        a.s += x == x ? 0.0f : x;        // a NaN beside nothing else
        return;
    }
    a.s = (a.m == m ? a.s : a.s * expf(a.m - m)) + expf(x - m);
    a.m = m;
}

template <typename T, int NT, int WORDS>
__global__ void __launch_bounds__(NT, NT * WORDS <= 2560 ? 2 : 1) k_distill(DistillArgs g) {
    constexpr int N = Word<T>::N;
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ float di_smem[];
    __shared__ float red[NT / 32];
    __shared__ Stat parts[NT / 32], mine;
    const Top t = {reinterpret_cast<int*>(di_smem), di_smem + g.top, di_smem + 2 * g.top};
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = (int)(blockIdx.x / C);
    const T* z = static_cast<const T*>(g.z) + (long long)row * g.ldz;
    T* grad = g.grad ? static_cast<T*>(g.grad) + (long long)row * g.ldg : nullptr;

    // this CTA's words of the row; entry e of the row is column e
    const int before = entries_before(z, g.vocab), words = (g.vocab - before) / N;
    const int share = (words + C - 1) / C, w0 = min(words, rank * share), w1 = min(words, w0 + share);
    const int behind = before + words * N;                       // the entries from here on go one by one
    const int c0 = rank == 0 ? 0 : before + w0 * N, c1 = rank == C - 1 ? g.vocab : before + w1 * N;
    Word<T> x[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        const int w = w0 + i * NT + (int)threadIdx.x;
        if (w < w1) x[i].w = __ldcs(reinterpret_cast<const uint4*>(z + before) + w);
    }
    // one entry a thread: before the words with the first CTA, behind them with the last
    int single = -1;
    if (rank == 0 && (int)threadIdx.x < before) single = threadIdx.x;
    const int back = NT - 1 - (int)threadIdx.x;                  // NT > two words' entries: another thread
    if (rank == C - 1 && behind + back < g.vocab) single = behind + back;
    const float xs = single >= 0 ? to_f32(z[single]) : -INFINITY;

    const bool any = teacher_side<NT>(g, row, t, red);
    // the logits at the ids: all of them for the loss, those of this CTA's columns
    // for the gradient (in place, others may be overwritten already)
    const int from = rank == 0 && !g.lse_in ? 0 : c0, to = rank == 0 && !g.lse_in ? g.vocab : c1;
    for (int k = threadIdx.x; k < g.top; k += NT) t.z[k] = t.id[k] >= from && t.id[k] < to ? to_f32(z[t.id[k]]) : 0.0f;

    const Exp<FAST> ex(g.inv_tau);
    float m, inv_s = 1.0f, lse;
    if (g.lse_in) {
        m = lse = g.lse_in[row];
        __syncthreads();
    } else {
        Stat a = {-INFINITY, 0.0f};
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
            float v[N];
            x[i].get(v);
            float top = v[0];
#pragma unroll
            for (int j = 1; j < N; ++j) top = fmaxf(top, v[j]);
            a.m = fmaxf(a.m, top);
        }
        a.m = fmaxf(a.m, xs);
        // a thread whose entries are all -Inf (or NaN) sums against 0
        const float base = a.m == -INFINITY ? 0.0f : a.m;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
            float v[N];
            x[i].get(v);
#pragma unroll
            for (int j = 0; j < N; ++j) a.s += ex.below(v[j], base);
        }
        a.s += ex.below(xs, base);
        a.m *= g.inv_tau;
        a = warp_join(a);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0) parts[warp] = a;
        __syncthreads();
        a = parts[0];
#pragma unroll
        for (int w = 1; w < NT / 32; ++w) a = join(a, parts[w]);
        if (C > 1) {
            if (threadIdx.x == 0) mine = a;
            cluster.sync();              // also: every CTA has gathered its entries, the row may be overwritten
            a = *cluster.map_shared_rank(&mine, 0);
            for (int r = 1; r < C; ++r) a = join(a, *cluster.map_shared_rank(&mine, r));
        }
        m = a.m;
        inv_s = 1.0f / a.s;
        lse = m + logf(a.s);
        if (rank == 0) {
            const float d = any ? divergence<NT>(g, t, lse, red) : 0.0f;
            if (threadIdx.x == 0) {
                g.loss[row] = any ? g.tau * g.tau * d : 0.0f;
                g.lse[row] = lse;
            }
        }
    }
    if (grad) {
        const float scale = any ? g.dloss[row] * g.tau : 0.0f;
        const float level = ex.level(m);
        auto q = [&](float v) { return ex.against(v, level) * inv_s; };      // (from lse alone: s = 1)
        uint4* out = reinterpret_cast<uint4*>(grad + before);
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const int w = w0 + i * NT + (int)threadIdx.x;
            if (w >= w1) continue;
            float v[N];
            x[i].get(v);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = any ? scale * q(v[j]) : 0.0f;
            x[i].set(v);
            __stcs(out + w, x[i].w);
        }
        if (single >= 0) from_f32(any ? scale * q(xs) : 0.0f, grad[single]);
        __syncthreads();
        if (any) put_right<NT>(g, t, grad, c0, c1, scale, q);
    }
    if (C > 1 && !g.lse_in) cluster.sync();      // the others have read this CTA's statistics
}

// Any row: one CTA, the logits read once for the statistics and once more for
// the gradient, entry by entry.
template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_long(DistillArgs g) {
    extern __shared__ float di_smem[];
    __shared__ float red[NT / 32];
    __shared__ Stat parts[NT / 32];
    const Top t = {reinterpret_cast<int*>(di_smem), di_smem + g.top, di_smem + 2 * g.top};
    const int row = (int)blockIdx.x;
    const T* z = static_cast<const T*>(g.z) + (long long)row * g.ldz;
    const bool any = teacher_side<NT>(g, row, t, red);
    for (int k = threadIdx.x; k < g.top; k += NT) t.z[k] = t.id[k] >= 0 ? to_f32(z[t.id[k]]) : 0.0f;
    float m, inv_s = 1.0f;
    if (g.lse_in) {
        m = g.lse_in[row];
        __syncthreads();
    } else {
        Stat a = {-INFINITY, 0.0f};
#pragma unroll 4
        for (int c = threadIdx.x; c < g.vocab; c += NT) add_one(a, to_f32(z[c]) * g.inv_tau);
        a = warp_join(a);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0) parts[warp] = a;
        __syncthreads();
        a = parts[0];
        for (int w = 1; w < NT / 32; ++w) a = join(a, parts[w]);
        m = a.m;
        inv_s = 1.0f / a.s;
        const float lse = m + logf(a.s), d = any ? divergence<NT>(g, t, lse, red) : 0.0f;
        if (threadIdx.x == 0) {
            g.loss[row] = any ? g.tau * g.tau * d : 0.0f;
            g.lse[row] = lse;
        }
    }
    if (!g.grad) return;
    T* grad = static_cast<T*>(g.grad) + (long long)row * g.ldg;
    const float scale = any ? g.dloss[row] * g.tau : 0.0f;
    auto q = [&](float v) { return expf(v * g.inv_tau - m) * inv_s; };
#pragma unroll 4
    for (int c = threadIdx.x; c < g.vocab; c += NT) from_f32(any ? scale * q(to_f32(z[c])) : 0.0f, grad[c]);
    __syncthreads();
    if (any) put_right<NT>(g, t, grad, 0, g.vocab, scale, q);
}

int check_distill(const iso_mat* z, const void* ids, int32_t ids_i64, const iso_mat* teacher, float tau,
                  const iso_mat* grad) {
    ISO_TRY(check_mat(z));
    ISO_TRY(check_mat(teacher));
    if (grad) ISO_TRY(check_mat(grad));
    if ((ids_i64 != 0 && ids_i64 != 1) || !(tau > 0.0f) || !std::isfinite(tau) || !std::isfinite(1.0f / tau)) return ISO_ERR_ARG;
    if (teacher->rows != z->rows || (grad && (grad->rows != z->rows || grad->cols != z->cols))) return ISO_ERR_SHAPE;
    if (grad && grad->dtype != z->dtype) return ISO_ERR_DTYPE;
    if (teacher->cols > ISO_DISTILL_MAX_TOP) return ISO_ERR_UNSUPPORTED;
    if (teacher->rows && teacher->cols) {
        if (!ids) return ISO_ERR_ARG;
        if (reinterpret_cast<uintptr_t>(ids) % (ids_i64 ? 8 : 4)) return ISO_ERR_ALIGN;
    }
    return ISO_OK;
}
Bytes2D flat(const void* p, uint64_t bytes) { return {reinterpret_cast<uintptr_t>(p), 1, bytes, bytes}; }

template <typename T, int NT, int WORDS>
int launch_rows(const DistillArgs& g, int cluster, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)g.rows * (unsigned)cluster);
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = (size_t)g.top * 12;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)cluster;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    TRAIN_LAUNCH(cudaLaunchKernelEx(&cfg, k_distill<T, NT, WORDS>, g));
    return ISO_OK;
}

template <typename T>
int launch_distill(const DistillArgs& g, cudaStream_t s) {
    constexpr int N = Word<T>::N;
    // words from the first boundary on must be words of the gradient too, in every row
    const bool alike = !g.grad || (((reinterpret_cast<uintptr_t>(g.z) ^ reinterpret_cast<uintptr_t>(g.grad)) & 15u) == 0 &&
                                   (g.rows == 1 || (g.ldz - g.ldg) * (long long)sizeof(T) % 16 == 0));
    const int words = g.vocab / N;
    if (!alike || words > DI_MAX_CLUSTER * 512 * DI_MAX_WORDS || (long long)g.rows * DI_MAX_CLUSTER > EXTENT_LIMIT) {
        TRAIN_LAUNCH((k_distill_long<T, 1024><<<(unsigned)g.rows, 1024, (size_t)g.top * 12, s>>>(g)));
        return ISO_OK;
    }
    if (words <= 128 * 4) return words <= 128 ? launch_rows<T, 128, 1>(g, 1, s) : launch_rows<T, 128, 4>(g, 1, s);
    // the smallest cluster that holds a row; larger ones while they leave SMs idle
    int C = 1;
    while (words > C * 512 * DI_MAX_WORDS) C *= 2;
    while (C < DI_MAX_CLUSTER && (long long)g.rows * C * 2 <= train_sms() && words > C * 512) C *= 2;
    const int need = (words + C * 512 - 1) / (C * 512);
    if (need <= 2) return launch_rows<T, 512, 2>(g, C, s);
    if (need <= 5) return launch_rows<T, 512, 5>(g, C, s);
    return launch_rows<T, 512, DI_MAX_WORDS>(g, C, s);
}

int run_distill(DistillArgs& g, const iso_mat* z, const void* ids, int32_t ids_i64, const iso_mat* teacher, float tau,
                const iso_mat* grad, int32_t* status, cudaStream_t s) {
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (z->rows == 0) return ISO_OK;
    g.z = z->data;
    g.ids = ids;
    g.teacher = teacher->data;
    g.grad = grad ? grad->data : nullptr;
    g.status = status;
    g.ldz = z->ld;
    g.ldt = teacher->ld;
    g.ldg = grad ? grad->ld : 0;
    g.rows = (int)z->rows;
    g.vocab = (int)z->cols;
    g.top = (int)teacher->cols;
    g.ids_i64 = ids_i64;
    g.teacher_f32 = teacher->dtype == ISO_F32;
    g.tau = tau;
    g.inv_tau = 1.0f / tau;
    return z->dtype == ISO_BF16 ? launch_distill<__nv_bfloat16>(g, s) : launch_distill<float>(g, s);
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_distill(const iso_mat* logits, const void* ids, int32_t ids_i64, const iso_mat* teacher,
                    float temperature, float* loss, float* lse, const float* dloss, const iso_mat* dlogits,
                    int32_t* status, void* stream) {
    ISO_TRY(check_distill(logits, ids, ids_i64, teacher, temperature, dlogits));
    const uint64_t n = (uint64_t)logits->rows;
    if (n && (!loss || !lse || (dlogits && !dloss))) return ISO_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(loss) | reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(dloss)) & 3u)
        return ISO_ERR_ALIGN;
    const Bytes2D outs[3] = {flat(loss, 4 * n), flat(lse, 4 * n), dlogits ? bytes_of(dlogits) : Bytes2D{}};
    const Bytes2D ins[4] = {bytes_of(logits), flat(ids, n * (uint64_t)teacher->cols * (ids_i64 ? 8 : 4)),
                            bytes_of(teacher), flat(dloss, dloss ? 4 * n : 0)};
    const bool in_place = dlogits && dlogits->data == logits->data && (dlogits->ld == logits->ld || n == 1);
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 4; ++i)
            if (!(o == 2 && i == 0 && in_place) && share_bytes(outs[o], ins[i])) return ISO_ERR_ARG;
        for (int p = 0; p < o; ++p)
            if (share_bytes(outs[o], outs[p])) return ISO_ERR_ARG;
    }
    DistillArgs g{};
    g.loss = loss;
    g.lse = lse;
    g.dloss = dloss;
    return run_distill(g, logits, ids, ids_i64, teacher, temperature, dlogits, status, static_cast<cudaStream_t>(stream));
}

int32_t iso_distill_grad(const float* dloss, const iso_mat* logits, const void* ids, int32_t ids_i64,
                         const iso_mat* teacher, float temperature, const float* lse, const iso_mat* dlogits,
                         int32_t* status, void* stream) {
    if (!dlogits) return ISO_ERR_ARG;
    ISO_TRY(check_distill(logits, ids, ids_i64, teacher, temperature, dlogits));
    const uint64_t n = (uint64_t)logits->rows;
    if (n && (!dloss || !lse)) return ISO_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(dloss)) & 3u) return ISO_ERR_ALIGN;
    const bool in_place = dlogits->data == logits->data && (dlogits->ld == logits->ld || n == 1);
    const Bytes2D out = bytes_of(dlogits);
    if ((!in_place && share_bytes(out, bytes_of(logits))) || share_bytes(out, bytes_of(teacher)) ||
        share_bytes(out, flat(ids, n * (uint64_t)teacher->cols * (ids_i64 ? 8 : 4))) ||
        share_bytes(out, flat(dloss, 4 * n)) || share_bytes(out, flat(lse, 4 * n)))
        return ISO_ERR_ARG;
    DistillArgs g{};
    g.dloss = dloss;
    g.lse_in = lse;
    return run_distill(g, logits, ids, ids_i64, teacher, temperature, dlogits, status, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
