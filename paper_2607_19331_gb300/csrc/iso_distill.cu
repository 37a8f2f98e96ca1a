// iso_distill.cu -- distillation from a teacher's top logits: loss, log-sum-exp
// and the gradient of the logits.
//
// The logits are all of the traffic (K ids and teacher logits a row against a
// vocabulary), and a row takes one exponential an entry for the sum and one for
// the gradient: bound by HBM.  Loss and gradient in one call therefore read the
// logits once:
//   k_distill       a cluster of 1 ... 8 CTAs holds a whole row in registers, as
//                   it was loaded (up to ten 16-byte words a thread), so every
//                   load of a row is in flight at once; statistics per warp, CTA
//                   and cluster (distributed shared memory), and the gradient
//                   from the same registers.  A warp of its own takes the
//                   teacher's side beside the loads: its softmax, the logits at
//                   its ids, the loss, and after the row the entries at the ids, each
//                   by the CTA that owns its column.
//   k_distill_long  rows that do not fit, or whose logits and gradient do not
//                   sit alike in 16-byte words: one CTA a row, two passes.
// A row off a 16-byte boundary is taken as its words from the first boundary on;
// the entries before and behind them (under one word each) go one by one.
// Statistics: a warp takes its maximum m and its sum of exp((x - m) / tau), and
// sums of several warps and CTAs are joined as sum of s_i exp((m_i - m) / tau), m
// the largest m_i, in a fixed order.  In the exponents m / tau is a level, rounded
// once, that lse takes back: exp(x / tau - level) then has one rounding, of a
// number that is small where the weight is not.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <cmath>

namespace iso {
namespace {

constexpr int DI_MAX_CLUSTER = 8;
constexpr int DI_MAX_WORDS = 10;         // 16-byte words of a row a thread holds
constexpr int DI_WARP_TOP = 128;         // up to this many slots the teacher's warp adds up equal ids alone
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
    int32_t ids_i64, teacher_f32, cluster;
    float tau, inv_tau;
};

// exp(x / tau - level): of a bf16 row by the hardware's exponential (2 ulp, far
// below the rounding of the gradient, and random beside one another in the sum) of
// base 2, of a binary32 row by expf.
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
    // of a maximum; 0 where there is none, so that -Inf weighs 0
    __device__ __forceinline__ float level(float m) const { return m == -INFINITY ? 0.0f : m * c; }
    __device__ __forceinline__ float level_of(float lse) const { return FAST ? lse * LOG2E : lse; }
    __device__ __forceinline__ float lse(float level, float s) const {
        return FAST ? (level + log2f(s)) * 0.6931471805599453f : level + logf(s);
    }
    __device__ __forceinline__ float at(float x, float level) const { return of(fmaf(x, c, -level)); }
};

// two at a time
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void parts_of(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// m: the largest entry (-Inf: none); s: the sum of exp(x / tau - level(m))
struct Stat {
    float m, s;
};
template <bool FAST>
__device__ __forceinline__ Stat join_lanes(Stat a, int lanes, const Exp<FAST>& ex) {     // of `lanes` lanes (a power of two)
    float m = a.m;
    for (int o = lanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float s = a.m == m ? a.s : a.s * ex.of(ex.level(a.m) - ex.level(m));
    if (a.m == -INFINITY) s = a.s;                  // 0, or NaN
    for (int o = lanes / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return {m, s};
}

__device__ __forceinline__ long long id_at(const DistillArgs& g, long long i) {
    return g.ids_i64 ? static_cast<const long long*>(g.ids)[i] : (long long)static_cast<const int*>(g.ids)[i];
}
__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}

// The teacher's side of a row, in shared memory of each CTA
struct Top {
    int* id;                 // -1: unused
    float* p;                // probabilities
    float* z;                // logits at the ids
    float* mass;             // probabilities of all slots of the id together
};
__device__ __forceinline__ Top top_of(float* smem, int n) {
    return {reinterpret_cast<int*>(smem), smem + n, smem + 2 * n, smem + 3 * n};
}
constexpr int DI_TOP_BYTES = 16;

__device__ __forceinline__ float mass_of(const Top& t, int top, int id) {
    float p = 0.0f;
    for (int j = 0; j < top; ++j) p += t.id[j] == id ? t.p[j] : 0.0f;
    return p;
}

// By one warp; z is read at the ids in [from, to).  Whether the row has a used slot
// with a weight (else its loss and gradient are 0).
template <typename T>
__device__ __forceinline__ bool teacher_side(const DistillArgs& g, int row, const T* z, const Top& t, int from, int to) {
    const int lane = threadIdx.x & 31;
    float m = -INFINITY;
    bool nan = false;
    for (int k = lane; k < g.top; k += 32) {
        const long long v = id_at(g, (long long)row * g.top + k), at = (long long)row * g.ldt + k;
        const bool used = v >= 0 && v < g.vocab;
        if (!used && v != -1 && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_INDEX);
        float x = -INFINITY;
        if (used)
            x = (g.teacher_f32 ? static_cast<const float*>(g.teacher)[at]
                               : __bfloat162float(static_cast<const __nv_bfloat16*>(g.teacher)[at])) * g.inv_tau;
        t.id[k] = used ? (int)v : -1;
        t.p[k] = x;
        t.z[k] = v >= from && v < to ? to_f32(z[v]) : 0.0f;
        m = fmaxf(m, x);
        nan |= x != x;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    nan = __any_sync(0xFFFFFFFFu, nan);
    if (m == -INFINITY && !nan) return false;
    float s = 0.0f;
    for (int k = lane; k < g.top; k += 32) {
        const float x = t.id[k] < 0 ? 0.0f : expf(t.p[k] - (nan ? __int_as_float(0x7FFFFFFF) : m));
        t.p[k] = x;
        s += x;
    }
    s = warp_sum(s);
    for (int k = lane; k < g.top; k += 32) t.p[k] = t.p[k] / s;
    __syncwarp();
    if (g.grad && g.top <= DI_WARP_TOP)
        for (int k = lane; k < g.top; k += 32) t.mass[k] = mass_of(t, g.top, t.id[k]);
    return true;
}

// sum_k p_k (log p_k - z_k / tau + lse), by one warp
__device__ __forceinline__ float divergence(const DistillArgs& g, const Top& t, float lse) {
    float s = 0.0f;
    for (int k = threadIdx.x & 31; k < g.top; k += 32) {
        const float p = t.p[k];
        if (t.id[k] >= 0 && p != 0.0f) s += p * (logf(p) - (t.z[k] * g.inv_tau - lse));
    }
    return warp_sum(s);
}

// The entries at the teacher's ids among columns [c0, c1), after the row: slots of
// one id write the same value.  q(z): scale times the student's probability.  By
// the whole CTA of `warps` warps, the last of them the teacher's.
template <typename T, typename Q>
__device__ __forceinline__ void put_right(const DistillArgs& g, const Top& t, T* grad, int c0, int c1, float scale, int warps, Q q) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (g.top <= DI_WARP_TOP) {
        if (warp != warps - 1) return;
        for (int k = lane; k < g.top; k += 32)
            if (t.id[k] >= c0 && t.id[k] < c1) from_f32(q(t.z[k]) - scale * t.mass[k], grad[t.id[k]]);
        return;
    }
    for (int k = warp; k < g.top; k += warps) {       // many slots: a warp adds up each id's
        const int id = t.id[k];
        if (id < c0 || id >= c1) continue;
        float p = 0.0f;
        for (int j = lane; j < g.top; j += 32) p += t.id[j] == id ? t.p[j] : 0.0f;
        p = warp_sum(p);
        if (lane == 0) from_f32(q(t.z[k]) - scale * p, grad[id]);
    }
}

template <typename T>
struct Word {                            // 16 bytes of a row
    static constexpr int N = 16 / sizeof(T);
    uint4 w;
    __device__ __forceinline__ void get(uint64_t (&v)[N / 2]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (sizeof(T) == 2) {
                float a, b;
                bf16x2_to_f32(u[i], a, b);
                v[i] = pair_of(a, b);
            } else {
                v[i] = pair_of(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
            }
        }
    }
    __device__ __forceinline__ void set(const uint64_t (&v)[N / 2]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            float a, b;
            parts_of(v[i], a, b);
            if constexpr (sizeof(T) == 2) u[i] = f32_to_bf16x2(a, b);
            else {
                u[2 * i] = __float_as_uint(a);
                u[2 * i + 1] = __float_as_uint(b);
            }
        }
        w = make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ __forceinline__ float top() const {      // a NaN counts as nothing
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
            const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
            return fmaxf(__low2float(m), __high2float(m));
        } else {
            return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
        }
    }
};

// Entries before a row's first 16-byte boundary (all of them for a shorter row)
template <typename T>
__device__ __forceinline__ int entries_before(const T* row, int n) {
    const int off = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / (int)sizeof(T);
    return min(off, n);
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int THREADS>
__device__ __forceinline__ void sync_some(int barrier) { asm volatile("bar.sync %0, %1;" :: "r"(barrier), "n"(THREADS) : "memory"); }
template <int THREADS>
__device__ __forceinline__ void arrive_some(int barrier) { asm volatile("bar.arrive %0, %1;" :: "r"(barrier), "n"(THREADS) : "memory"); }

// NT threads hold the row, 32 more are the teacher's.  The row does not wait for
// the teacher's side, a chain of loads, before its own entries are out: a row
// without any is cleared afterwards.  Only in place the gradient waits until the
// logits at the ids have been read.
template <typename T, int NT, int WORDS>
__global__ void __launch_bounds__(NT + 32, NT == 512 ? 2 : NT == 256 ? 4 : 6) k_distill(const __grid_constant__ DistillArgs g) {
    constexpr int N = Word<T>::N, WARPS = NT / 32;
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ float di_smem[];
    __shared__ Stat parts[WARPS], of_cta[DI_MAX_CLUSTER];
    __shared__ int any_s;
    const Top t = top_of(di_smem, g.top);
    const int C = g.cluster, rank = C > 1 ? (int)(blockIdx.x % C) : 0;
    const int row = (int)(blockIdx.x / C), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool joint = g.lse_in == nullptr;
    if (C > 1 && joint) cluster_arrive();
    const T* z = static_cast<const T*>(g.z) + (long long)row * g.ldz;
    T* grad = g.grad ? static_cast<T*>(g.grad) + (long long)row * g.ldg : nullptr;
    const bool in_place = g.grad == g.z;
    const Exp<FAST> ex(g.inv_tau);

    // this CTA's words of the row; entry e of the row is column e
    const int before = entries_before(z, g.vocab), words = (g.vocab - before) / N;
    const int share = (words + C - 1) / C, w0 = min(words, rank * share), w1 = min(words, w0 + share);
    const int behind = before + words * N;                       // the entries from here on go one by one
    const int c0 = rank == 0 ? 0 : before + w0 * N, c1 = rank == C - 1 ? g.vocab : before + w1 * N;
    // of the CTA's partial sums: the cluster's maximum (as a level) and sum
    auto all_of = [&](Stat a) {
        a.m = __shfl_sync(0xFFFFFFFFu, a.m, 0);
        a.s = __shfl_sync(0xFFFFFFFFu, a.s, 0);
        return a;
    };
    auto of_warps = [&] {
        Stat a = {-INFINITY, 0.0f};
        if (lane < WARPS) a = parts[lane];
        return all_of(join_lanes(a, WARPS, ex));
    };
    auto of_ctas = [&] {
        Stat a = {-INFINITY, 0.0f};
        if (lane < C) a = of_cta[lane];
        return all_of(join_lanes(a, DI_MAX_CLUSTER, ex));
    };
    const float dloss = grad ? g.dloss[row] : 0.0f;
    const float lse_in = joint ? 0.0f : g.lse_in[row];
    float level = 0.0f, by = 0.0f, xs = -INFINITY;
    int single = -1;
    if (warp < WARPS) {
        Word<T> x[WORDS];
        const uint4* at = reinterpret_cast<const uint4*>(z + before) + w0 + threadIdx.x;
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            if (w0 + i * NT + (int)threadIdx.x < w1) x[i].w = __ldcs(at + i * NT);
        // one entry a thread: before the words with the first CTA, behind them with the last
        if (rank == 0 && (int)threadIdx.x < before) single = threadIdx.x;
        const int back = NT - 1 - (int)threadIdx.x;              // NT > two words' entries: another thread
        if (rank == C - 1 && behind + back < g.vocab) single = behind + back;
        if (single >= 0) xs = to_f32(z[single]);
        float inv_s = 1.0f;
        if (joint) {
            Stat a = {xs, 0.0f};
#pragma unroll
            for (int i = 0; i < WORDS; ++i)
                if (w0 + i * NT + (int)threadIdx.x < w1) a.m = fmaxf(a.m, x[i].top());
            if (a.m != a.m) a.m = -INFINITY;                     // (xs alone may be NaN)
#pragma unroll
            for (int o = 16; o; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xFFFFFFFFu, a.m, o));
            level = ex.level(a.m);
            const uint64_t cc = pair_of(ex.c, ex.c), ll = pair_of(-level, -level);
            uint64_t sum = pair_of(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
                uint64_t v[N / 2];
                x[i].get(v);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) {
                    float p, q;
                    parts_of(fma2(v[j], cc, ll), p, q);
                    sum = add2(sum, pair_of(ex.of(p), ex.of(q)));
                }
            }
            float p, q;
            parts_of(sum, p, q);
            a.s = warp_sum(p + q + (single >= 0 ? ex.at(xs, level) : 0.0f));
            if (lane == 0) parts[warp] = a;
            if (C == 1) arrive_some<NT + 32>(2);                 // for the teacher's warp
            if (C > 1 || grad) {
                sync_some<NT>(1);
                a = of_warps();
            }
            if (C > 1) {
                cluster_wait();          // every CTA of the cluster runs
                if (warp == 0 && lane < C) {
                    uint32_t to;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&of_cta[rank])), "r"(lane));
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(to), "f"(a.m), "f"(a.s) : "memory");
                }
                __syncwarp();
                cluster_arrive();
                cluster_wait();
                a = of_ctas();
            } else if (in_place) {
                sync_some<NT + 32>(3);   // the logits at the ids have been read
            }
            level = ex.level(a.m);
            inv_s = 1.0f / a.s;
        } else {
            level = ex.level_of(lse_in);
            if (in_place) sync_some<NT + 32>(3);
        }
        by = dloss * g.tau * inv_s;
        if (grad) {
            const uint64_t cc = pair_of(ex.c, ex.c), ll = pair_of(-level, -level), bb = pair_of(by, by);
            uint4* out = reinterpret_cast<uint4*>(grad + before) + w0 + threadIdx.x;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
                uint64_t v[N / 2];
                x[i].get(v);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) {
                    float p, q;
                    parts_of(fma2(v[j], cc, ll), p, q);
                    v[j] = mul2(pair_of(ex.of(p), ex.of(q)), bb);
                }
                x[i].set(v);
                __stcs(out + i * NT, x[i].w);
            }
            if (single >= 0) from_f32(by * ex.at(xs, level), grad[single]);
        }
    } else {
        if (C > 1 && joint) {
            cluster_wait();
            if (!in_place) cluster_arrive();
        }
        // the logits at the ids: all of them for the loss, those of this CTA's columns
        // for the gradient (in place, others may be overwritten already)
        const bool all = rank == 0 && joint;
        const bool any = (grad || rank == 0) && teacher_side(g, row, z, t, all ? 0 : c0, all ? g.vocab : c1);
        if (lane == 0) any_s = any;
        if (C > 1 && joint) {
            if (in_place) cluster_arrive();
            cluster_wait();
        } else if (in_place) {
            sync_some<NT + 32>(3);
        }
        if (joint) {
            if (C == 1) sync_some<NT + 32>(2);
            const Stat a = C > 1 ? of_ctas() : of_warps();
            level = ex.level(a.m);
            by = dloss * g.tau / a.s;
            if (rank == 0) {
                const float lse = a.m == -INFINITY && a.s == 0.0f ? -INFINITY : ex.lse(level, a.s);
                const float d = any ? divergence(g, t, lse) : 0.0f;
                if (lane == 0) {
                    g.loss[row] = any ? g.tau * g.tau * d : 0.0f;
                    g.lse[row] = lse;
                }
            }
        } else {
            level = ex.level_of(lse_in);
            by = dloss * g.tau;
        }
    }
    if (!grad) return;
    __syncthreads();
    if (any_s) {
        put_right(g, t, grad, c0, c1, dloss * g.tau, WARPS + 1, [&](float v) { return by * ex.at(v, level); });
    } else {
        for (int c = c0 + (int)threadIdx.x; c < c1; c += NT + 32) from_f32(0.0f, grad[c]);
    }
}

// Any row: one CTA, the logits read once for the statistics and once more for
// the gradient, entry by entry.
template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_long(const __grid_constant__ DistillArgs g) {
    constexpr int WARPS = NT / 32;
    extern __shared__ float di_smem[];
    __shared__ Stat parts[WARPS];
    __shared__ int any_s;
    const Top t = top_of(di_smem, g.top);
    const int row = (int)blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* z = static_cast<const T*>(g.z) + (long long)row * g.ldz;
    const Exp<false> ex(g.inv_tau);
    if (warp == WARPS - 1) {
        const bool any = teacher_side(g, row, z, t, 0, g.vocab);
        if (lane == 0) any_s = any;
    }
    Stat a = {-INFINITY, 0.0f};
    if (!g.lse_in) {
#pragma unroll 8
        for (int c = threadIdx.x; c < g.vocab; c += NT) a.m = fmaxf(a.m, to_f32(z[c]));
#pragma unroll
        for (int o = 16; o; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xFFFFFFFFu, a.m, o));
        const float level = ex.level(a.m);
#pragma unroll 8
        for (int c = threadIdx.x; c < g.vocab; c += NT) a.s += ex.at(to_f32(z[c]), level);
        a.s = warp_sum(a.s);
        if (lane == 0) parts[warp] = a;
    }
    __syncthreads();
    const bool any = any_s;
    float level, inv_s = 1.0f;
    if (g.lse_in) {
        level = ex.level_of(g.lse_in[row]);
    } else {
        a = {-INFINITY, 0.0f};
        if (lane < WARPS) a = parts[lane];
        a = join_lanes(a, WARPS, ex);
        level = ex.level(a.m);
        inv_s = 1.0f / a.s;
        if (warp == WARPS - 1) {
            const float lse = a.m == -INFINITY && a.s == 0.0f ? -INFINITY : ex.lse(level, a.s);
            const float d = any ? divergence(g, t, lse) : 0.0f;
            if (lane == 0) {
                g.loss[row] = any ? g.tau * g.tau * d : 0.0f;
                g.lse[row] = lse;
            }
        }
    }
    if (!g.grad) return;
    T* grad = static_cast<T*>(g.grad) + (long long)row * g.ldg;
    const float scale = any ? g.dloss[row] * g.tau : 0.0f, by = scale * inv_s;
#pragma unroll 8
    for (int c = threadIdx.x; c < g.vocab; c += NT) from_f32(any ? by * ex.at(to_f32(z[c]), level) : 0.0f, grad[c]);
    __syncthreads();
    if (any) put_right(g, t, grad, 0, g.vocab, scale, WARPS, [&](float v) { return by * ex.at(v, level); });
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
int launch_rows(DistillArgs g, int cluster, cudaStream_t s) {
    g.cluster = cluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)g.rows * (unsigned)cluster);
    cfg.blockDim = dim3(NT + 32);
    cfg.dynamicSmemBytes = (size_t)g.top * DI_TOP_BYTES;
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
        TRAIN_LAUNCH((k_distill_long<T, 1024><<<(unsigned)g.rows, 1024, (size_t)g.top * DI_TOP_BYTES, s>>>(g)));
        return ISO_OK;
    }
    if (words <= 128 * 4) return words <= 128 ? launch_rows<T, 128, 1>(g, 1, s) : launch_rows<T, 128, 4>(g, 1, s);
    if (words > DI_MAX_CLUSTER * 256 * DI_MAX_WORDS) return launch_rows<T, 512, DI_MAX_WORDS>(g, DI_MAX_CLUSTER, s);
    // the smallest cluster that holds a row; larger ones while they leave SMs idle
    int C = 1;
    while (words > C * 256 * DI_MAX_WORDS) C *= 2;
    while (C < DI_MAX_CLUSTER && (long long)g.rows * C * 2 <= train_sms() && words > C * 256) C *= 2;
    return words <= C * 256 * 5 ? launch_rows<T, 256, 5>(g, C, s) : launch_rows<T, 256, DI_MAX_WORDS>(g, C, s);
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
