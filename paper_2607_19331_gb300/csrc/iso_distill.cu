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
//   k_distill_stream  the same for many long rows, by clusters that stay.
//   k_distill_long  rows that do not fit, or whose logits and gradient do not
//                   sit alike in 16-byte words: one CTA a row, two passes.
// A row off a 16-byte boundary is taken as its words from the first boundary on;
// the entries before and behind them (under one word each) go one by one.
// Statistics: a warp takes its maximum m and its sum of exp((x - m) / tau), and
// sums of several warps and CTAs are joined as sum of s_i exp((m_i - m) / tau), m
// the largest m_i, in a fixed order.  Exponents are (x - m) / tau, not x / tau -
// m / tau: the rounding of m / tau is as large as any number where logits are (masks of
// -1e10 or of the type's lowest value), and such a warp's sum, whose weight is 0,
// would be infinite.  For the same reason the loss takes z - m and log s, not
// z / tau - lse.  From lse alone a probability is held at 1, whatever lse was rounded to.
#include "iso_tc.cuh"
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

namespace iso {
namespace {

constexpr int DI_MAX_CLUSTER = 8;
constexpr int DI_MAX_WORDS = 10;         // 16-byte words of a row a thread holds
constexpr int DI_WARP_TOP = 256;         // up to this many slots the teacher's warp adds up equal ids alone
using tc::LOG2E;
using tc::pair_of;
using tc::parts_of;
using tc::fma2;
using tc::add2;
using tc::mul2;

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
    int32_t stages, share;               // k_distill_stream: rows in flight, words of a row a CTA has room for
    float tau, inv_tau;
    uint64_t wait_ns;
};

// What exponents are formed from: a maximum m (exp((x - m) / tau)) or lse
struct Ref {
    float by, minus;
};
// exp((x - m) / tau): of a bf16 row by the hardware's exponential (2 ulp, far
// below the rounding of the gradient, and random beside one another in the sum) of
// base 2, of a binary32 row by expf.
template <bool FAST>
struct Exp {
    float c, inv_tau;
    __device__ __forceinline__ explicit Exp(float inv_tau) : c(FAST ? inv_tau * LOG2E : inv_tau), inv_tau(inv_tau) {}
    __device__ __forceinline__ float of(float x) const {
        if constexpr (FAST) {
            float y;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
            return y;
        } else {
            return expf(x);
        }
    }
    // of a maximum; of 0 where there is none, so that -Inf weighs 0
    __device__ __forceinline__ Ref from_max(float m) const { return {c, m == -INFINITY ? 0.0f : -m}; }
    __device__ __forceinline__ Ref from_lse(float lse) const { return {inv_tau, -lse}; }
    template <bool LSE>
    __device__ __forceinline__ float at(float x, Ref r) const {
        if constexpr (LSE) {
            const float e = fmaf(x, r.by, r.minus);
            return of(min0(FAST ? e * LOG2E : e));              // at most 1 however lse was rounded
        } else {
            return of((x + r.minus) * r.by);
        }
    }
    static __device__ __forceinline__ float min0(float x) {     // a NaN stays one
        float y;
        asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(0.0f));
        return y;
    }
};
// The same of two entries at a time
template <bool FAST, bool LSE>
struct ExpPair {
    uint64_t by, minus, scale;
    const Exp<FAST>& ex;
    __device__ __forceinline__ ExpPair(const Exp<FAST>& ex, Ref r)
        : by(pair_of(r.by, r.by)), minus(pair_of(r.minus, r.minus)), scale(pair_of(LOG2E, LOG2E)), ex(ex) {}
    __device__ __forceinline__ uint64_t of(uint64_t x) const {
        float p, q;
        uint64_t e = LSE ? fma2(x, by, minus) : mul2(add2(x, minus), by);
        if constexpr (LSE && FAST) e = mul2(e, scale);
        parts_of(e, p, q);
        if constexpr (LSE) {
            p = ex.min0(p);
            q = ex.min0(q);
        }
        return pair_of(ex.of(p), ex.of(q));
    }
};

// m: the largest entry (-Inf: none); s: the sum of exp((x - m) / tau)
struct Stat {
    float m, s;
};
template <bool FAST>
__device__ __forceinline__ Stat join_lanes(Stat a, int lanes, const Exp<FAST>& ex) {     // of `lanes` lanes (a power of two)
    float m = a.m;
    for (int o = lanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float s = a.m == m ? a.s : a.s * ex.of((a.m - m) * ex.c);
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
    uint16_t* bucket;        // of ids, by a hash: the slot of one, or DI_SEVERAL
};
constexpr int DI_BUCKET_BITS = 11;
constexpr uint16_t DI_SEVERAL = 0xFFFF;
constexpr int top_floats(int n) { return 4 * n + (1 << DI_BUCKET_BITS) / 2; }
__device__ __forceinline__ Top top_of(float* smem, int n) {
    return {reinterpret_cast<int*>(smem), smem + n, smem + 2 * n, smem + 3 * n, reinterpret_cast<uint16_t*>(smem + 4 * n)};
}

// p of every slot's id, by one warp.  An id that shares its bucket with no other slot's
// has that slot alone; for the few others the warp goes through all slots.  (All slots
// against all: 200 slots of 4096 rows of 152064 cost 370 us more than 64.)
__device__ __forceinline__ void masses(const Top& t, int top) {
    const int lane = threadIdx.x & 31;
    auto bucket_of = [&](int id) { return (uint32_t)id * 2654435761u >> (32 - DI_BUCKET_BITS); };
    for (int k = lane; k < top; k += 32)
        if (t.id[k] >= 0) t.bucket[bucket_of(t.id[k])] = (uint16_t)k;
    __syncwarp();
    for (int k = lane; k < top; k += 32)
        if (t.id[k] >= 0 && t.bucket[bucket_of(t.id[k])] != k) t.bucket[bucket_of(t.id[k])] = DI_SEVERAL;
    __syncwarp();
    for (int k0 = 0; k0 < top; k0 += 32) {
        const int k = k0 + lane, id = k < top ? t.id[k] : -1;
        float mass = id >= 0 ? t.p[k] : 0.0f;
        unsigned several = __ballot_sync(0xFFFFFFFFu, id >= 0 && t.bucket[bucket_of(id)] == DI_SEVERAL);
        while (several) {
            const int l = __ffs(several) - 1;
            several &= several - 1;
            const int want = __shfl_sync(0xFFFFFFFFu, id, l);
            float p = 0.0f;
            for (int j = lane; j < top; j += 32) p += t.id[j] == want ? t.p[j] : 0.0f;
            p = warp_sum(p);
            if (lane == l) mass = p;
        }
        if (k < top) t.mass[k] = mass;
    }
}

// By one warp; z is read at the ids in [from, to).  Whether the row has a used slot
// with a weight (else its loss and gradient are 0).
template <typename T>
__device__ __forceinline__ bool teacher_side(const DistillArgs& g, int row, const T* z, const Top& t, int from, int to) {
    const int lane = threadIdx.x & 31;
    float m = -INFINITY;
    bool nan = false;
    constexpr int EACH = 4;                      // slots a lane reads at once: ids and teacher's logits, then z
    for (int k0 = lane; k0 < g.top; k0 += 32 * EACH) {
        long long v[EACH];
        float x[EACH], y[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int k = k0 + 32 * i;
            const long long at = (long long)row * g.ldt + k;
            v[i] = -1;
            x[i] = y[i] = 0.0f;
            if (k < g.top) {
                v[i] = id_at(g, (long long)row * g.top + k);
                x[i] = g.teacher_f32 ? static_cast<const float*>(g.teacher)[at]
                                     : __bfloat162float(static_cast<const __nv_bfloat16*>(g.teacher)[at]);
            }
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (v[i] >= from && v[i] < to) y[i] = to_f32(z[v[i]]);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int k = k0 + 32 * i;
            if (k >= g.top) continue;
            const bool used = v[i] >= 0 && v[i] < g.vocab;
            if (!used && v[i] != -1 && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_INDEX);
            const float w = used ? x[i] : -INFINITY;
            t.id[k] = used ? (int)v[i] : -1;
            t.p[k] = w;
            t.z[k] = y[i];
            m = fmaxf(m, w);
            nan |= w != w;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    nan = __any_sync(0xFFFFFFFFu, nan);
    if (m == -INFINITY && !nan) return false;
    float s = 0.0f;
    for (int k = lane; k < g.top; k += 32) {
        const float x = t.id[k] < 0 ? 0.0f : expf((t.p[k] - (nan ? __int_as_float(0x7FFFFFFF) : m)) * g.inv_tau);
        t.p[k] = x;
        s += x;
    }
    s = warp_sum(s);
    for (int k = lane; k < g.top; k += 32) t.p[k] = t.p[k] / s;
    __syncwarp();
    if (g.grad && g.top <= DI_WARP_TOP) masses(t, g.top);
    return true;
}

// tau^2 sum_k p_k (log p_k - log q_k), log q = (z - m) / tau - log s, by one warp
__device__ __forceinline__ float divergence(const DistillArgs& g, const Top& t, float m, float log_s) {
    const float tau = g.tau;
    float s = 0.0f;
    for (int k = threadIdx.x & 31; k < g.top; k += 32) {
        const float p = t.p[k];
        if (t.id[k] >= 0 && p != 0.0f) s += p * (tau * (logf(p) + log_s) - (t.z[k] - m));
    }
    return tau * warp_sum(s);
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
// 128 threads for short rows (4096 x 4000 bf16 with its gradient: 18 us, 256 threads 28;
// 4096 x 2000 f32: 20, 29), five words a thread where they hold the row (2000 x 8000 bf16:
// 16.4 us, ten 18.2), larger clusters while rows leave SMs idle (8 x 32000 f32: 4.8 us, one
// no larger than needed 5.5).
template <typename T, int NT, int WORDS, bool LSE>
__global__ void __launch_bounds__(NT + 32, NT == 512 ? 2 : NT == 256 ? 4 : 6) k_distill(const __grid_constant__ DistillArgs g) {
    constexpr int N = Word<T>::N, WARPS = NT / 32;
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ float di_smem[];
    __shared__ Stat parts[WARPS], of_cta[DI_MAX_CLUSTER];
    __shared__ int any_s;
    const Top t = top_of(di_smem, g.top);
    const int C = g.cluster, rank = C > 1 ? (int)(blockIdx.x % C) : 0;
    const int row = (int)(blockIdx.x / C), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr bool joint = !LSE;
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
    // of the CTA's partial sums: the cluster's maximum and sum
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
    Ref ref = {};
    float by = 0.0f, xs = -INFINITY;
    auto weight = [&](float x) { return ex.template at<LSE>(x, ref); };
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
        __syncwarp();            // every load is issued before the first is used (4096 x 50000 f32, loss: 345 -> 309 us)
        float inv_s = 1.0f;
        if (joint) {
            Stat a = {xs, 0.0f};
#pragma unroll
            for (int i = 0; i < WORDS; ++i)
                if (w0 + i * NT + (int)threadIdx.x < w1) a.m = fmaxf(a.m, x[i].top());
            if (a.m != a.m) a.m = -INFINITY;                     // (xs alone may be NaN)
#pragma unroll
            for (int o = 16; o; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xFFFFFFFFu, a.m, o));
            ref = ex.from_max(a.m);
            const ExpPair<FAST, false> two(ex, ref);
            uint64_t sum = pair_of(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
                uint64_t v[N / 2];
                x[i].get(v);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) sum = add2(sum, two.of(v[j]));
            }
            float p, q;
            parts_of(sum, p, q);
            a.s = warp_sum(p + q + (single >= 0 ? weight(xs) : 0.0f));
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
            ref = ex.from_max(a.m);
            inv_s = 1.0f / a.s;
        } else {
            ref = ex.from_lse(lse_in);
            if (in_place) sync_some<NT + 32>(3);
        }
        by = dloss * g.tau * inv_s;
        if (grad) {
            const ExpPair<FAST, LSE> two(ex, ref);
            const uint64_t bb = pair_of(by, by);
            uint4* out = reinterpret_cast<uint4*>(grad + before) + w0 + threadIdx.x;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if (w0 + i * NT + (int)threadIdx.x >= w1) continue;
                uint64_t v[N / 2];
                x[i].get(v);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) v[j] = mul2(two.of(v[j]), bb);
                x[i].set(v);
                __stcs(out + i * NT, x[i].w);
            }
            if (single >= 0) from_f32(by * weight(xs), grad[single]);
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
            ref = ex.from_max(a.m);
            by = dloss * g.tau / a.s;
            if (rank == 0) {
                const float log_s = logf(a.s), lse = a.m == -INFINITY && a.s == 0.0f ? -INFINITY : fmaf(a.m, g.inv_tau, log_s);
                const float d = any ? divergence(g, t, a.m, log_s) : 0.0f;
                if (lane == 0) {
                    g.loss[row] = d;
                    g.lse[row] = lse;
                }
            }
        } else {
            ref = ex.from_lse(lse_in);
            by = dloss * g.tau;
        }
    }
    if (!grad) return;
    __syncthreads();
    if (any_s) {
        put_right(g, t, grad, c0, c1, dloss * g.tau, WARPS + 1, [&](float v) { return by * weight(v); });
    } else {
        for (int c = c0 + (int)threadIdx.x; c < c1; c += NT + 32) from_f32(0.0f, grad[c]);
    }
}

// Many long rows: the cluster stays and goes from row to row (by the number of
// clusters), its words of the next rows on their way into shared memory by bulk
// copies meanwhile, so that no load waits for a row's exchanges, nor a row for a
// launch.  A row: its words summed up, the cluster's exchange of sums, its words again for
// the gradient.  Four warps take the teacher's side of every fourth row each, a
// chain of loads that is as long as two rows.  Bound by HBM where a row fits one
// CTA, and for the gradient alone (6.3 TB/s); with larger clusters by the exchange, whose
// latency no other row of the cluster covers.
// Measured against k_distill, loss with gradient / loss / gradient alone, us:
//   4096 x 152064 bf16 (clusters of 4)   527 / 360 / 395   against 524 / 313 / 378
//   4096 x 76032 bf16 (2)                256 / 175 / 205   against 265 / 156 / 191
//   4096 x 50000 f32 (2)                 321 / 203 / 267   against 444 / 309 / 294
//   4096 x 50000 bf16 (1)                130 /  79 / 139   against 219 / 144 / 151
//   8192 x 32000 bf16 (1)                187 / 120 / 176   against 253 / 150 / 197
//   8192 x 20000 bf16 (1)                161 / 103 / 108   against 132 /  65 / 125
//   8192 x 12000 bf16 (1)                145 /  89 /  81   against  98 /  55 /  79
//   1024 x 50000 bf16 (1)                 42 /  25 /  41   against  58 /  41 /  41
//   600 x 152064 bf16 (4)                 88 /  61 /  69   against  80 /  52 /  58
//   1024 x 76032 f32 (4)                 150 / 104 / 109   against 135 /  90 /  94
// so it takes rows of DS_MIN_WORDS that fit one CTA, DS_ROUNDS rows for each, and rows of
// larger clusters for a gradient, DS_ROUNDS_CLUSTER for each (clusters of 8 for the first case: 913).  (The words kept in
// registers from the first pass on, with 20 a thread: 589 us for the first case.)
constexpr int DS_NT = 256, DS_TEACHERS = 4, DS_MAX_STAGES = 4, DS_SMEM = 220 * 1024;
constexpr int DS_MIN_WORDS = 3000, DS_ROUNDS = 4, DS_ROUNDS_CLUSTER = 32;
__device__ __forceinline__ bool probe_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
template <typename T, bool LSE>
__global__ void __launch_bounds__(DS_NT + 32 * DS_TEACHERS, 1) k_distill_stream(const __grid_constant__ DistillArgs g) {
    constexpr int NT = DS_NT, N = Word<T>::N, WARPS = NT / 32;
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ __align__(128) unsigned char ds_smem[];
    __shared__ Stat parts[WARPS], of_cta[2][DI_MAX_CLUSTER], of_row[DS_TEACHERS];
    __shared__ __align__(8) uint64_t full[DS_MAX_STAGES], exchanged[2], prepared[DS_TEACHERS], written[DS_TEACHERS];
    __shared__ volatile int any_s[DS_TEACHERS];
    __shared__ volatile int gave_up;
    __shared__ int first_bad;                    // rows of this cluster from here on are not whole
    const int C = g.cluster, rank = (int)(blockIdx.x % C), clusters = (int)(gridDim.x / C), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t stage_bytes = (size_t)g.share * 16;
    float* const tops = reinterpret_cast<float*>(ds_smem + g.stages * stage_bytes);
    const Exp<FAST> ex(g.inv_tau);
    const tc::Waits wait = {g.wait_ns, &gave_up};

    // this CTA's part of a row, as in k_distill
    struct Part {
        const T* z;
        int before, w0, w1, behind, c0, c1;
    };
    auto part_of = [&](int row) {
        Part p;
        p.z = static_cast<const T*>(g.z) + (long long)row * g.ldz;
        p.before = entries_before(p.z, g.vocab);
        const int words = (g.vocab - p.before) / N, share = (words + C - 1) / C;
        p.w0 = min(words, rank * share);
        p.w1 = min(words, p.w0 + share);
        p.behind = p.before + words * N;
        p.c0 = rank == 0 ? 0 : p.before + p.w0 * N;
        p.c1 = rank == C - 1 ? g.vocab : p.before + p.w1 * N;
        return p;
    };
    int issued = 0;                              // copies: the i-th into stage i mod stages
    auto copy = [&](int row, int stage) {        // by one thread
        if (row >= g.rows || gave_up) return;
        ++issued;
        const Part p = part_of(row);
        const uint32_t bar = smem_u32(&full[stage]), bytes = (uint32_t)(p.w1 - p.w0) * 16u;
        if (bytes == 0) {
            mbar_arrive(bar);
            return;
        }
        mbar_arrive_tx(bar, bytes);
        bulk_g2s(smem_u32(ds_smem + stage * stage_bytes), p.z + p.before + (long long)p.w0 * N, bytes, bar);
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < g.stages; ++i) mbar_init(smem_u32(&full[i]), 1);
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&exchanged[i]), (uint32_t)C);
        for (int i = 0; i < DS_TEACHERS; ++i) {
            mbar_init(smem_u32(&prepared[i]), 1);
            mbar_init(smem_u32(&written[i]), WARPS);
        }
        gave_up = 0;
        first_bad = INT_MAX;
        mbar_fence_init();
    }
    __syncthreads();
    if (C > 1) {
        cluster_arrive();
        cluster_wait();                          // every CTA of the cluster runs, its barriers are there
    }
    const int row0 = (int)(blockIdx.x / C);
    if (warp < WARPS) {
        if (threadIdx.x == 0)
            for (int i = 0; i < g.stages; ++i) copy(row0 + i * clusters, i);
        int stage = 0, it = 0;
        uint32_t parity = 0;
        for (int row = row0; row < g.rows; row += clusters, ++it) {
            const int slot = it % DS_TEACHERS, b = it & 1;
            const Part p = part_of(row);
            T* const grad = g.grad ? static_cast<T*>(g.grad) + (long long)row * g.ldg : nullptr;
            const float dloss = grad ? g.dloss[row] : 0.0f;
            const bool stop = gave_up;           // after a give-up no row is whole: its stage may hold an earlier one
            Ref ref = ex.from_lse(LSE ? g.lse_in[row] : 0.0f);
            float inv_s = 1.0f;
            const uint4* const words = reinterpret_cast<const uint4*>(ds_smem + stage * stage_bytes);
            int single = -1;
            if (rank == 0 && (int)threadIdx.x < p.before) single = threadIdx.x;
            const int back = NT - 1 - (int)threadIdx.x;
            if (rank == C - 1 && p.behind + back < g.vocab) single = p.behind + back;
            const float xs = single >= 0 ? to_f32(p.z[single]) : -INFINITY;
            bool whole = wait.warp(smem_u32(&full[stage]), parity);
            const int n = p.w1 - p.w0;
            Stat a = {xs, 0.0f};
            if (!LSE) {
#pragma unroll 4
                for (int i = threadIdx.x; i < n; i += NT) {
                    Word<T> x;
                    x.w = words[i];
                    a.m = fmaxf(a.m, x.top());
                }
                if (a.m != a.m) a.m = -INFINITY;
#pragma unroll
                for (int o = 16; o; o >>= 1) a.m = fmaxf(a.m, __shfl_xor_sync(0xFFFFFFFFu, a.m, o));
                ref = ex.from_max(a.m);
                const ExpPair<FAST, false> two(ex, ref);
                uint64_t sum = pair_of(0.0f, 0.0f);
#pragma unroll 4
                for (int i = threadIdx.x; i < n; i += NT) {
                    Word<T> x;
                    x.w = words[i];
                    uint64_t v[N / 2];
                    x.get(v);
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) sum = add2(sum, two.of(v[j]));
                }
                float s0, s1;
                parts_of(sum, s0, s1);
                a.s = warp_sum(s0 + s1 + (single >= 0 ? ex.template at<false>(xs, ref) : 0.0f));
                whole = __all_sync(0xFFFFFFFFu, whole && !stop);
                if (lane == 0) parts[warp] = whole ? a : Stat{a.m, __int_as_float(0x7FFFFFFF)};
                sync_some<NT>(1);
                a = {-INFINITY, 0.0f};
                if (lane < WARPS) a = parts[lane];
                a = join_lanes(a, WARPS, ex);
                a.m = __shfl_sync(0xFFFFFFFFu, a.m, 0);
                a.s = __shfl_sync(0xFFFFFFFFu, a.s, 0);
                if (C > 1) {
                    if (warp == 0) {
                        // this CTA's teacher's side has read the logits at its ids
                        whole = whole && wait.warp(smem_u32(&prepared[slot]), (uint32_t)(it / DS_TEACHERS) & 1u);
                        if (!whole) a.m = a.s = __int_as_float(0x7FFFFFFF);      // for every CTA
                        if (lane < C) {
                            uint32_t to, at;
                            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&of_cta[b][rank])), "r"(lane));
                            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&exchanged[b])), "r"(lane));
                            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(to), "f"(a.m), "f"(a.s) : "memory");
                            asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(at) : "memory");
                        }
                        __syncwarp();
                    }
                    const uint32_t ph = (uint32_t)(it >> 1) & 1u;
                    if (whole && !__all_sync(0xFFFFFFFFu, probe_cluster(smem_u32(&exchanged[b]), ph)))
                        whole = wait.warp(smem_u32(&exchanged[b]), ph) && __all_sync(0xFFFFFFFFu, probe_cluster(smem_u32(&exchanged[b]), ph));
                    a = {-INFINITY, 0.0f};
                    if (lane < C) a = of_cta[b][lane];
                    a = join_lanes(a, DI_MAX_CLUSTER, ex);
                    a.m = __shfl_sync(0xFFFFFFFFu, a.m, 0);
                    a.s = __shfl_sync(0xFFFFFFFFu, a.s, 0);
                }
                ref = ex.from_max(a.m);
                inv_s = 1.0f / a.s;
            }
            if (LSE) whole = __all_sync(0xFFFFFFFFu, whole && !stop);
            whole = whole && wait.warp(smem_u32(&prepared[slot]), (uint32_t)(it / DS_TEACHERS) & 1u);
            if (!whole && lane == 0) {
                gave_up = 1;
                atomicMin(&first_bad, it);
            }
            // (not before: until then the slot's warp may be reading those of its last row)
            if (threadIdx.x == 0 && !LSE && whole) of_row[slot] = a;
            if (grad && whole) {                 // (in place, what is not whole may still be read as logits)
                const bool any = any_s[slot];
                const float by = dloss * g.tau * inv_s;
                const ExpPair<FAST, LSE> two(ex, ref);
                const uint64_t bb = pair_of(by, by);
                uint4* const out = reinterpret_cast<uint4*>(grad + p.before) + p.w0;
#pragma unroll 4
                for (int i = threadIdx.x; i < n; i += NT) {
                    Word<T> x;
                    x.w = words[i];
                    uint64_t v[N / 2];
                    x.get(v);
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) v[j] = mul2(two.of(v[j]), bb);
                    x.set(v);
                    if (!any) x.w = make_uint4(0u, 0u, 0u, 0u);
                    __stcs(out + i, x.w);
                }
                if (single >= 0) from_f32(any ? by * ex.template at<LSE>(xs, ref) : 0.0f, grad[single]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&written[slot]));
            sync_some<NT>(1);                    // the row's place may be filled again
            if (threadIdx.x == 0) copy(row + g.stages * clusters, stage);
            if (++stage == g.stages) {
                stage = 0;
                parity ^= 1u;
            }
        }
        if (threadIdx.x == 0) {
            // no copy is in flight when the CTA ends, after a give-up either
            for (int i = max(0, issued - g.stages); i < issued; ++i)
                wait.drain(smem_u32(&full[i % g.stages]), (uint32_t)(i / g.stages) & 1u);
        }
    } else {
        const int slot = warp - WARPS;
        const Top t = top_of(tops + slot * top_floats(g.top), g.top);
        int it = slot;
        uint32_t ph = 0;
        for (int row = row0 + slot * clusters; row < g.rows; row += DS_TEACHERS * clusters, it += DS_TEACHERS, ph ^= 1u) {
            const Part p = part_of(row);
            bool any = false;
            const bool all = rank == 0 && !LSE;
            if (g.grad || rank == 0) any = teacher_side(g, row, p.z, t, all ? 0 : p.c0, all ? g.vocab : p.c1);
            if (lane == 0) any_s[slot] = any;
            tc::arrive_warp(smem_u32(&prepared[slot]));
            const float dloss = g.grad ? g.dloss[row] : 0.0f;
            Ref ref = ex.from_lse(LSE ? g.lse_in[row] : 0.0f);
            float by = dloss * g.tau;
            if (!wait.warp(smem_u32(&written[slot]), ph) || *static_cast<volatile int*>(&first_bad) <= it) {
                if (lane == 0) atomicMin(&first_bad, it);
                break;
            }
            if (!LSE) {
                const Stat a = of_row[slot];
                ref = ex.from_max(a.m);
                by = dloss * g.tau / a.s;
                if (rank == 0) {
                    const float log_s = logf(a.s), lse = a.m == -INFINITY && a.s == 0.0f ? -INFINITY : fmaf(a.m, g.inv_tau, log_s);
                    const float d = any ? divergence(g, t, a.m, log_s) : 0.0f;
                    if (lane == 0) {
                        g.loss[row] = d;
                        g.lse[row] = lse;
                    }
                }
            }
            if (g.grad && any)
                for (int k = lane; k < g.top; k += 32)
                    if (t.id[k] >= p.c0 && t.id[k] < p.c1)
                        from_f32(by * ex.template at<LSE>(t.z[k], ref) - dloss * g.tau * t.mass[k],
                                 static_cast<T*>(g.grad)[(long long)row * g.ldg + t.id[k]]);
            __syncwarp();
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (first_bad != INT_MAX) {
        // what a give-up left unfinished, in this CTA's columns; where it came before a
        // row's sums went out, the cluster's other CTAs have NaN from those
        for (long long row = row0 + (long long)first_bad * clusters; row < g.rows; row += clusters) {
            const Part p = part_of((int)row);
            if (g.grad)
                for (int c = p.c0 + (int)threadIdx.x; c < p.c1; c += NT + 32 * DS_TEACHERS)
                    from_f32(__int_as_float(0x7FFFFFFF), static_cast<T*>(g.grad)[row * g.ldg + c]);
            if (!LSE && rank == 0 && threadIdx.x == 0) g.loss[row] = g.lse[row] = __int_as_float(0x7FFFFFFF);
        }
    }
    if (C > 1) {
        cluster_arrive();
        cluster_wait();                          // the other CTAs' sums for this one have come
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
        const Ref origin = ex.from_max(a.m);
#pragma unroll 8
        for (int c = threadIdx.x; c < g.vocab; c += NT) a.s += ex.at<false>(to_f32(z[c]), origin);
        a.s = warp_sum(a.s);
        if (lane == 0) parts[warp] = a;
    }
    __syncthreads();
    const bool any = any_s;
    Ref ref;
    float inv_s = 1.0f;
    if (g.lse_in) {
        ref = ex.from_lse(g.lse_in[row]);
    } else {
        a = {-INFINITY, 0.0f};
        if (lane < WARPS) a = parts[lane];
        a = join_lanes(a, WARPS, ex);
        ref = ex.from_max(a.m);
        inv_s = 1.0f / a.s;
        if (warp == WARPS - 1) {
            const float log_s = logf(a.s), lse = a.m == -INFINITY && a.s == 0.0f ? -INFINITY : fmaf(a.m, g.inv_tau, log_s);
            const float d = any ? divergence(g, t, a.m, log_s) : 0.0f;
            if (lane == 0) {
                g.loss[row] = d;
                g.lse[row] = lse;
            }
        }
    }
    if (!g.grad) return;
    T* grad = static_cast<T*>(g.grad) + (long long)row * g.ldg;
    const float scale = any ? g.dloss[row] * g.tau : 0.0f, by = scale * inv_s;
    auto weight = [&](float x) { return g.lse_in ? ex.at<true>(x, ref) : ex.at<false>(x, ref); };
#pragma unroll 8
    for (int c = threadIdx.x; c < g.vocab; c += NT) from_f32(any ? by * weight(to_f32(z[c])) : 0.0f, grad[c]);
    __syncthreads();
    if (any) put_right(g, t, grad, 0, g.vocab, scale, WARPS, [&](float v) { return by * weight(v); });
}

int check_distill(const iso_mat* z, const void* ids, int32_t ids_i64, const iso_mat* teacher, float tau,
                  const iso_mat* grad) {
    ISO_TRY(check_mat(z));
    ISO_TRY(check_mat(teacher));
    if (grad) ISO_TRY(check_mat(grad));
    if ((ids_i64 != 0 && ids_i64 != 1) || !(tau > 0.0f) || !std::isfinite(tau) || !std::isfinite(1.0f / tau * LOG2E)) return ISO_ERR_ARG;
    if (teacher->rows != z->rows || (grad && (grad->rows != z->rows || grad->cols != z->cols))) return ISO_ERR_SHAPE;
    if (grad && grad->dtype != z->dtype) return ISO_ERR_DTYPE;
    if (teacher->cols > ISO_DISTILL_MAX_TOP) return ISO_ERR_UNSUPPORTED;
    if (teacher->rows && teacher->cols) {
        if (!ids) return ISO_ERR_ARG;
        if (reinterpret_cast<uintptr_t>(ids) % (ids_i64 ? 8 : 4)) return ISO_ERR_ALIGN;
    }
    return ISO_OK;
}
constexpr uint64_t DISTILL_WAIT_NS = 2000000000;   // a wait gives up after this long, unless told otherwise
std::atomic<uint64_t> g_distill_wait_ns{DISTILL_WAIT_NS};

Bytes2D flat(const void* p, uint64_t bytes) { return {reinterpret_cast<uintptr_t>(p), 1, bytes, bytes}; }

template <typename T, int NT, int WORDS>
int launch_rows(DistillArgs g, int cluster, cudaStream_t s) {
    g.cluster = cluster;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)g.rows * (unsigned)cluster);
    cfg.blockDim = dim3(NT + 32);
    cfg.dynamicSmemBytes = (size_t)top_floats(g.top) * 4;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)cluster;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    TRAIN_LAUNCH(g.lse_in ? cudaLaunchKernelEx(&cfg, k_distill<T, NT, WORDS, true>, g) : cudaLaunchKernelEx(&cfg, k_distill<T, NT, WORDS, false>, g));
    return ISO_OK;
}

// clusters that run at once on the current device
template <typename T, bool LSE>
int resident_clusters(int cluster, size_t smem) {
    static std::atomic<int> known[64][4];        // [device][log2 cluster]
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    const int at = cluster == 1 ? 0 : cluster == 2 ? 1 : cluster == 4 ? 2 : 3;
    n = known[dev][at].load(std::memory_order_relaxed);
    if (n) return n;
    if (cudaFuncSetAttribute(k_distill_stream<T, LSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, DS_SMEM) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(train_sms() / cluster * cluster));
    cfg.blockDim = dim3(DS_NT + 32 * DS_TEACHERS);
    cfg.dynamicSmemBytes = DS_SMEM;
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeClusterDimension;
    a.val.clusterDim.x = (unsigned)cluster;
    a.val.clusterDim.y = a.val.clusterDim.z = 1;
    cfg.attrs = &a;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, k_distill_stream<T, LSE>, &cfg) != cudaSuccess || n <= 0) return 0;
    known[dev][at].store(n, std::memory_order_relaxed);
    return n;
}
template <typename T, bool LSE>
int launch_stream(DistillArgs g, int cluster, int share, cudaStream_t s) {
    const size_t tops = DS_TEACHERS * (size_t)top_floats(g.top) * 4;
    g.cluster = cluster;
    g.share = (share + 7) / 8 * 8;               // (stages on 128-byte boundaries)
    g.stages = (int)std::min<size_t>(DS_MAX_STAGES, (DS_SMEM - tops) / ((size_t)g.share * 16));
    const int n = resident_clusters<T, LSE>(cluster, DS_SMEM);
    if (n <= 0) return ISO_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<long long>(g.rows, n) * (unsigned)cluster);
    cfg.blockDim = dim3(DS_NT + 32 * DS_TEACHERS);
    cfg.dynamicSmemBytes = DS_SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)cluster;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    TRAIN_LAUNCH(cudaLaunchKernelEx(&cfg, k_distill_stream<T, LSE>, g));
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
        TRAIN_LAUNCH((k_distill_long<T, 1024><<<(unsigned)g.rows, 1024, (size_t)top_floats(g.top) * 4, s>>>(g)));
        return ISO_OK;
    }
    if (words <= 128 * 4) return words <= 128 ? launch_rows<T, 128, 1>(g, 1, s) : launch_rows<T, 128, 4>(g, 1, s);
    if (words > DI_MAX_CLUSTER * 256 * DI_MAX_WORDS) return launch_rows<T, 512, DI_MAX_WORDS>(g, DI_MAX_CLUSTER, s);
    // streamed (up to DI_WARP_TOP slots, which a teacher's warp handles alone): the rule
    // stands with k_distill_stream
    if (g.top <= DI_WARP_TOP && words >= DS_MIN_WORDS) {
        const long long room = (DS_SMEM - DS_TEACHERS * 4LL * top_floats(g.top)) / 2 / 16;       // words a CTA can hold of two rows
        int C = 1;
        while (C < DI_MAX_CLUSTER && words > C * room) C *= 2;
        const long long rounds = C == 1 ? DS_ROUNDS : DS_ROUNDS_CLUSTER;
        if (words <= C * room && (C == 1 || g.grad) && (long long)g.rows * C >= rounds * train_sms())
            return g.lse_in ? launch_stream<T, true>(g, C, (words + C - 1) / C, s) : launch_stream<T, false>(g, C, (words + C - 1) / C, s);
    }
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
    g.wait_ns = g_distill_wait_ns.load(std::memory_order_relaxed);
    return z->dtype == ISO_BF16 ? launch_distill<__nv_bfloat16>(g, s) : launch_distill<float>(g, s);
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int64_t iso_distill_wait_ns(int64_t ns) {
    return (int64_t)(ns < 0 ? g_distill_wait_ns.load(std::memory_order_relaxed)
                            : g_distill_wait_ns.exchange((uint64_t)ns, std::memory_order_relaxed));
}

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
