// iso_attn_simt.cuh -- attention and its gradients on the CUDA cores, a tile of 64
// rows by 256 threads: any type, head dimension, stride and alignment, in
// binary32 throughout.  Tiles of 64 x 64 in shared memory as binary32; a thread
// has 4 x 4 of S and 4 x (dim / 16) of a sum.  A product takes two 16-byte shared
// loads per sixteen multiply-adds and is bound by those.
//
// What a query does not see is not multiplied at all, so a NaN or an infinity there has no
// part.  The tensor-core kernels multiply it by a weight of 0, which is the same
// unless it is not finite; then their sums are not finite either, and they do the
// rows over with these functions.
#pragma once

#include "iso_attn.cuh"

namespace iso {
namespace {

constexpr int SA_B = 64;                 // rows and columns of a tile
constexpr int SA_TPB = 256;
constexpr int SA_PP = SA_B + 4;          // row of a P tile: no bank twice in eight lanes' 16-byte loads

template <int DP>
constexpr int sa_pitch() { return DP + 4; }
// shared memory of the tiles' functions below: operand tiles, weights
template <int DP>
constexpr int sa_smem(int tiles, int weights) { return (tiles * SA_B * sa_pitch<DP>() + weights * SA_B * SA_PP + 2 * SA_B) * 4; }

// the 256 threads of a tile, which may be part of a larger block
__device__ __forceinline__ void sa_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// rows row0 .. row0 + 63 of a head into shared memory; `valid` of them exist,
// the others and channels past dim are 0
template <typename T, int DP>
__device__ __forceinline__ void sa_load(float* s, const void* base, long long ld, long long row0, int valid, int col0, int dim) {
    const T* const from = static_cast<const T*>(base) + row0 * ld + col0;
    if (dim % 4 == 0 && ((reinterpret_cast<uintptr_t>(from) | (uintptr_t)(ld * (long long)sizeof(T))) & (4 * sizeof(T) - 1)) == 0) {
        // four channels a load
#pragma unroll 4
        for (int i = threadIdx.x; i < SA_B * DP / 4; i += SA_TPB) {
            const int r = i / (DP / 4), d = (i - r * (DP / 4)) * 4;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (r < valid && d < dim) {
                if constexpr (sizeof(T) == 4) {
                    v = *reinterpret_cast<const float4*>(from + r * ld + d);
                } else {
                    const uint2 w = *reinterpret_cast<const uint2*>(from + r * ld + d);
                    bf16x2_to_f32(w.x, v.x, v.y);
                    bf16x2_to_f32(w.y, v.z, v.w);
                }
            }
            *reinterpret_cast<float4*>(s + r * sa_pitch<DP>() + d) = v;
        }
        return;
    }
#pragma unroll 4
    for (int i = threadIdx.x; i < SA_B * DP; i += SA_TPB) {
        const int r = i / DP, d = i - r * DP;
        s[r * sa_pitch<DP>() + d] = r < valid && d < dim ? to_f32(from[r * ld + d]) : 0.0f;
    }
}

// acc[i][j] = A[ty + 16 i] . B[tx + 16 j]
template <int DP>
__device__ __forceinline__ void sa_dot(const float* a, const float* b, int ty, int tx, float (&acc)[4][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
#pragma unroll 2
    for (int d = 0; d < DP; d += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = *reinterpret_cast<const float4*>(a + (ty + 16 * i) * sa_pitch<DP>() + d);
            y[i] = *reinterpret_cast<const float4*>(b + (tx + 16 * i) * sa_pitch<DP>() + d);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
                acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
                acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
                acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
            }
    }
}

// acc[i][4 j + c] += sum_k P[ty + 16 i][k] V[k][4 tx + 64 j + c], k over the
// columns [lo[i], hi[i]) of each row: what is masked is not multiplied, so a NaN
// there stays out
template <int DP>
__device__ __forceinline__ void sa_mul(const float* p, const float* v, int ty, int tx, const int (&lo)[4], const int (&hi)[4],
                                       float (&acc)[4][DP / 16]) {
    const bool full = lo[0] <= 0 && lo[1] <= 0 && lo[2] <= 0 && lo[3] <= 0 && hi[0] >= SA_B && hi[1] >= SA_B &&
                      hi[2] >= SA_B && hi[3] >= SA_B;
    auto go = [&](auto masked) {
#pragma unroll 1
        for (int k = 0; k < SA_B; k += 4) {
            float4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(p + (ty + 16 * i) * SA_PP + k);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int j = 0; j < DP / 64; ++j) {
                    const float4 x = *reinterpret_cast<const float4*>(v + (k + c) * sa_pitch<DP>() + 4 * tx + 64 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float s = c == 0 ? w[i].x : c == 1 ? w[i].y : c == 2 ? w[i].z : w[i].w;
                        if (!decltype(masked)::value || (k + c >= lo[i] && k + c < hi[i])) {
                            acc[i][4 * j] = fmaf(s, x.x, acc[i][4 * j]);
                            acc[i][4 * j + 1] = fmaf(s, x.y, acc[i][4 * j + 1]);
                            acc[i][4 * j + 2] = fmaf(s, x.z, acc[i][4 * j + 2]);
                            acc[i][4 * j + 3] = fmaf(s, x.w, acc[i][4 * j + 3]);
                        }
                    }
                }
            }
        }
    };
    if (full) go(std::false_type{});
    else go(std::true_type{});
}

template <typename T, int DP>
__device__ __forceinline__ void sa_store(void* base, long long ld, long long row0, int valid, int col0, int dim, int ty, int tx,
                                         const float (&acc)[4][DP / 16], const float (&by)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty + 16 * i;
        if (r >= valid) continue;
        T* o = static_cast<T*>(base) + (row0 + r) * ld + col0;
#pragma unroll
        for (int j = 0; j < DP / 64; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int d = 4 * tx + 64 * j + c;
                if (d < dim) from_f32(acc[i][4 * j + c] * by[i], o[d]);
            }
    }
}

__device__ __forceinline__ float row_max(float x) {      // over the 16 lanes of a row
#pragma unroll
    for (int o = 8; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// out and lse of 64 queries (from t.first on) of head h over the keys [begin, end),
// into rows of their own matrix and vector; with `sums` a row's maximum and sum
// instead of lse
template <typename T, int DP, typename O>
__device__ __noinline__ void simt_attn(const AttnArgs& g, const AttnTile& t, int h, int begin, int end, O* out, long long ldo,
                                       float* lse, float* smem, float* sums = nullptr) {
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sq = smem, *const sk = sq + TILE, *const sv = sk + TILE, *const sp = sv + TILE;
    const int kh = h / g.group, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int rows = min(SA_B, t.nq - t.first);
    sa_load<T, DP>(sq, g.q, g.ldq, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim);
    int lo[4], hi[4], first, last, unused;
    float m[4], l[4], acc[4][DP / 16] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        attn_keys_of(g, t, t.first + min(ty + 16 * i, rows - 1), lo[i], hi[i]);
        lo[i] = max(lo[i], begin);
        hi[i] = min(hi[i], end);
        m[i] = -INFINITY;
        l[i] = 0.0f;
    }
    attn_keys_of(g, t, t.first, first, unused);
    attn_keys_of(g, t, t.first + rows - 1, unused, last);
    first = max(first, begin);
    last = min(last, end);
    for (int k0 = first / SA_B * SA_B; k0 < last; k0 += SA_B) {
        const int keys = min(SA_B, t.nk - k0);
        sa_sync();
        sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_sync();
        float s[4][4];
        sa_dot<DP>(sq, sk, ty, tx, s);
        int a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = lo[i] - k0;
            b[i] = hi[i] - k0;
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = tx + 16 * j;
                s[i][j] = c >= a[i] && c < b[i] ? s[i][j] * g.scale : -INFINITY;
                top = fmaxf(top, s[i][j]);
            }
            const float to = fmaxf(m[i], row_max(top));
            const float base = to == -INFINITY ? 0.0f : to, by = expf(m[i] - base);     // 0 before the first seen key
            m[i] = to;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = expf(s[i][j] - base);
                sp[(ty + 16 * i) * SA_PP + tx + 16 * j] = p;
                sum += p;
            }
            l[i] = l[i] * by + row_sum(sum);
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) acc[i][c] *= by;
        }
        sa_sync();
        sa_mul<DP>(sp, sv, ty, tx, a, b, acc);
    }
    float inv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        inv[i] = l[i] == 0.0f ? 0.0f : 1.0f / l[i];
        const int r = ty + 16 * i;
        if (tx == 0 && r < rows) {
            const long long at = (long long)h * g.q_rows + t.q0 + t.first + r;
            lse[at] = sums ? m[i] : m[i] + logf(l[i]);
            if (sums) sums[at] = l[i];
        }
    }
    sa_store<O, DP>(out, ldo, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim, ty, tx, acc, inv);
}

// dk and dv of 64 keys (from t.first on) of key head kh, over the query heads
// h0 .. h1 - 1, into rows of their own matrices
template <typename T, int DP, typename O>
__device__ __noinline__ void simt_grad_kv(const AttnArgs& g, const AttnTile& t, int kh, int h0, int h1, O* dk, long long lddk, O* dv,
                                          long long lddv, float* smem) {
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sk = smem, *const sv = sk + TILE, *const sq = sv + TILE, *const sd = sq + TILE, *const sp = sd + TILE,
                 *const ss = sp + SA_B * SA_PP, *const lse = ss + SA_B * SA_PP, *const delta = lse + SA_B;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int keys = min(SA_B, t.nk - t.first);
    sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim);
    sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim);
    int lo[4], hi[4], first, last, unused;
    float ak[4][DP / 16] = {}, av[4][DP / 16] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) attn_queries_of(g, t, t.first + min(ty + 16 * i, keys - 1), lo[i], hi[i]);
    attn_queries_of(g, t, t.first, first, unused);
    attn_queries_of(g, t, t.first + keys - 1, unused, last);
    for (int h = h0; h < h1; ++h) {
        for (int q0 = first / SA_B * SA_B; q0 < last; q0 += SA_B) {
            const int rows = min(SA_B, t.nq - q0);
            sa_sync();
            sa_load<T, DP>(sq, g.q, g.ldq, (long long)t.q0 + q0, rows, h * g.head_dim, g.head_dim);
            sa_load<T, DP>(sd, g.dout, g.lddo, (long long)t.q0 + q0, rows, h * g.head_dim, g.head_dim);
            if (threadIdx.x < SA_B) {
                const long long at = (long long)h * g.q_rows + t.q0 + q0 + threadIdx.x;
                lse[threadIdx.x] = (int)threadIdx.x < rows ? g.lse[at] : 0.0f;
                delta[threadIdx.x] = (int)threadIdx.x < rows ? g.delta[at] : 0.0f;
            }
            sa_sync();
            float s[4][4], dp[4][4];
            sa_dot<DP>(sk, sq, ty, tx, s);
            sa_dot<DP>(sv, sd, ty, tx, dp);
            int a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = lo[i] - q0;
                b[i] = hi[i] - q0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = tx + 16 * j;
                    const bool seen = c >= a[i] && c < b[i];
                    const float p = seen ? expf(s[i][j] * g.scale - lse[c]) : 0.0f;
                    sp[(ty + 16 * i) * SA_PP + c] = p;
                    ss[(ty + 16 * i) * SA_PP + c] = seen ? p * (dp[i][j] - delta[c]) : 0.0f;
                }
            }
            sa_sync();
            sa_mul<DP>(sp, sd, ty, tx, a, b, av);
            sa_mul<DP>(ss, sq, ty, tx, a, b, ak);
        }
    }
    const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f}, scale[4] = {g.scale, g.scale, g.scale, g.scale};
    sa_store<O, DP>(dk, lddk, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim, ty, tx, ak, scale);
    sa_store<O, DP>(dv, lddv, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim, ty, tx, av, one);
}

// dq of 64 queries (from t.first on) of head h
template <typename T, int DP>
__device__ __noinline__ void simt_grad_q(const AttnArgs& g, const AttnTile& t, int h, float* smem) {
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sq = smem, *const sd = sq + TILE, *const sk = sd + TILE, *const sv = sk + TILE, *const ss = sv + TILE;
    const int kh = h / g.group, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int rows = min(SA_B, t.nq - t.first);
    sa_load<T, DP>(sq, g.q, g.ldq, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim);
    sa_load<T, DP>(sd, g.dout, g.lddo, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim);
    int lo[4], hi[4], first, last, unused;
    float lse[4], delta[4], acc[4][DP / 16] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = min(ty + 16 * i, rows - 1);
        attn_keys_of(g, t, t.first + r, lo[i], hi[i]);
        const long long at = (long long)h * g.q_rows + t.q0 + t.first + r;
        lse[i] = g.lse[at];
        delta[i] = g.delta[at];
    }
    attn_keys_of(g, t, t.first, first, unused);
    attn_keys_of(g, t, t.first + rows - 1, unused, last);
    for (int k0 = first / SA_B * SA_B; k0 < last; k0 += SA_B) {
        const int keys = min(SA_B, t.nk - k0);
        sa_sync();
        sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_sync();
        float s[4][4], dp[4][4];
        sa_dot<DP>(sq, sk, ty, tx, s);
        sa_dot<DP>(sd, sv, ty, tx, dp);
        int a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = lo[i] - k0;
            b[i] = hi[i] - k0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = tx + 16 * j;
                const bool seen = c >= a[i] && c < b[i];
                ss[(ty + 16 * i) * SA_PP + c] = seen ? expf(s[i][j] * g.scale - lse[i]) * (dp[i][j] - delta[i]) : 0.0f;
            }
        }
        sa_sync();
        sa_mul<DP>(ss, sk, ty, tx, a, b, acc);
    }
    const float scale[4] = {g.scale, g.scale, g.scale, g.scale};
    sa_store<T, DP>(g.dq, g.lddq, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim, ty, tx, acc, scale);
}

}  // namespace
}  // namespace iso
