// iso_attn.cu -- attention and its gradients: entry points, and the kernels on
// the CUDA cores.
//
// Forward: one pass over the keys with the running maximum m and sum l of the
// softmax: O <- O e^(m - m') + e^(S - m') V.  Backward: the weights again from
// lse, P = e^(S - lse), and no atomics: k_simt_grad_kv owns a tile of keys and
// goes over the queries (of all query heads of its key head), k_simt_grad_q owns
// a tile of queries and goes over the keys; S and dP are formed in both (seven
// products instead of five), and every sum has a fixed order.
//
// The CUDA-core kernels take any type, head dimension, stride and alignment, in
// binary32 throughout: tiles of 64 x 64 in shared memory as binary32, 256 threads
// with 4 x 4 of S and 4 x (dim / 16) of a sum each.  A product takes two 16-byte
// shared loads per sixteen multiply-adds and is bound by those.
#include "iso_attn.cuh"

#include <algorithm>
#include <cmath>

namespace iso {
namespace {

constexpr int SA_B = 64;                 // rows and columns of a tile
constexpr int SA_TPB = 256;
constexpr int SA_PP = SA_B + 4;          // row of a P tile: no bank twice in eight lanes' 16-byte loads

template <int DP>
constexpr int sa_pitch() { return DP + 4; }

// rows row0 .. row0 + 63 of a head into shared memory; `valid` of them exist,
// the others and channels past dim are 0
template <typename T, int DP>
__device__ __forceinline__ void sa_load(float* s, const void* base, long long ld, long long row0, int valid, int col0, int dim) {
    for (int i = threadIdx.x; i < SA_B * DP; i += SA_TPB) {
        const int r = i / DP, d = i - r * DP;
        s[r * sa_pitch<DP>() + d] =
            r < valid && d < dim ? to_f32(static_cast<const T*>(base)[(row0 + r) * ld + col0 + d]) : 0.0f;
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

template <typename T, int DP>
__global__ void __launch_bounds__(SA_TPB) k_simt_attn(AttnArgs g) {
    extern __shared__ __align__(16) float sa_smem[];
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sq = sa_smem, *const sk = sq + TILE, *const sv = sk + TILE, *const sp = sv + TILE;
    const int h = blockIdx.x % g.heads, kh = h / g.group, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / g.heads, SA_B, false, t)) return;
    const int rows = min(SA_B, t.nq - t.first);
    sa_load<T, DP>(sq, g.q, g.ldq, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim);
    int lo[4], hi[4], first, last, unused;
    float m[4], l[4], acc[4][DP / 16] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        attn_keys_of(g, t, t.first + min(ty + 16 * i, rows - 1), lo[i], hi[i]);
        m[i] = -INFINITY;
        l[i] = 0.0f;
    }
    attn_keys_of(g, t, t.first, first, unused);
    attn_keys_of(g, t, t.first + rows - 1, unused, last);
    for (int k0 = first / SA_B * SA_B; k0 < last; k0 += SA_B) {
        const int keys = min(SA_B, t.nk - k0);
        __syncthreads();
        sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        __syncthreads();
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
        __syncthreads();
        sa_mul<DP>(sp, sv, ty, tx, a, b, acc);
    }
    float inv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        inv[i] = l[i] == 0.0f ? 0.0f : 1.0f / l[i];
        const int r = ty + 16 * i;
        if (tx == 0 && r < rows) g.lse[(long long)h * g.q_rows + t.q0 + t.first + r] = m[i] + logf(l[i]);
    }
    sa_store<T, DP>(const_cast<void*>(g.out), g.ldo, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim, ty, tx, acc, inv);
}

// delta[h][i] = sum_d dout_id out_id: a warp per row and head
template <typename T>
__global__ void __launch_bounds__(256) k_attn_delta(AttnArgs g) {
    const long long i = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (i >= (long long)g.q_rows * g.heads) return;
    const long long row = i / g.heads;
    const int h = (int)(i - row * g.heads);
    const T* o = static_cast<const T*>(g.out) + row * g.ldo + (long long)h * g.head_dim;
    const T* d = static_cast<const T*>(g.dout) + row * g.lddo + (long long)h * g.head_dim;
    float s = 0.0f;
    for (int c = lane; c < g.head_dim; c += 32) s = fmaf(to_f32(o[c]), to_f32(d[c]), s);
#pragma unroll
    for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
    if (lane == 0) g.delta[(long long)h * g.q_rows + row] = s;
}

// dk and dv of 64 keys of one key head
template <typename T, int DP>
__global__ void __launch_bounds__(SA_TPB) k_simt_grad_kv(AttnArgs g) {
    extern __shared__ __align__(16) float sa_smem[];
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sk = sa_smem, *const sv = sk + TILE, *const sq = sv + TILE, *const sd = sq + TILE, *const sp = sd + TILE,
                 *const ss = sp + SA_B * SA_PP;
    __shared__ float lse[SA_B], delta[SA_B];
    const int kv_heads = g.heads / g.group, kh = blockIdx.x % kv_heads, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / kv_heads, SA_B, true, t)) return;
    const int keys = min(SA_B, t.nk - t.first);
    sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim);
    sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim);
    int lo[4], hi[4], first, last, unused;
    float ak[4][DP / 16] = {}, av[4][DP / 16] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) attn_queries_of(g, t, t.first + min(ty + 16 * i, keys - 1), lo[i], hi[i]);
    attn_queries_of(g, t, t.first, first, unused);
    attn_queries_of(g, t, t.first + keys - 1, unused, last);
    for (int h = kh * g.group; h < (kh + 1) * g.group; ++h) {
        for (int q0 = first / SA_B * SA_B; q0 < last; q0 += SA_B) {
            const int rows = min(SA_B, t.nq - q0);
            __syncthreads();
            sa_load<T, DP>(sq, g.q, g.ldq, (long long)t.q0 + q0, rows, h * g.head_dim, g.head_dim);
            sa_load<T, DP>(sd, g.dout, g.lddo, (long long)t.q0 + q0, rows, h * g.head_dim, g.head_dim);
            if (threadIdx.x < SA_B) {
                const long long at = (long long)h * g.q_rows + t.q0 + q0 + threadIdx.x;
                lse[threadIdx.x] = (int)threadIdx.x < rows ? g.lse[at] : 0.0f;
                delta[threadIdx.x] = (int)threadIdx.x < rows ? g.delta[at] : 0.0f;
            }
            __syncthreads();
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
            __syncthreads();
            sa_mul<DP>(sp, sd, ty, tx, a, b, av);
            sa_mul<DP>(ss, sq, ty, tx, a, b, ak);
        }
    }
    const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f}, scale[4] = {g.scale, g.scale, g.scale, g.scale};
    sa_store<T, DP>(g.dk, g.lddk, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim, ty, tx, ak, scale);
    sa_store<T, DP>(g.dv, g.lddv, (long long)t.k0 + t.first, keys, kh * g.head_dim, g.head_dim, ty, tx, av, one);
}

// dq of 64 queries of one head
template <typename T, int DP>
__global__ void __launch_bounds__(SA_TPB) k_simt_grad_q(AttnArgs g) {
    extern __shared__ __align__(16) float sa_smem[];
    constexpr int TILE = SA_B * sa_pitch<DP>();
    float *const sq = sa_smem, *const sd = sq + TILE, *const sk = sd + TILE, *const sv = sk + TILE, *const ss = sv + TILE;
    const int h = blockIdx.x % g.heads, kh = h / g.group, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    AttnTile t;
    if (!attn_find_tile(g, blockIdx.x / g.heads, SA_B, false, t)) return;
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
        __syncthreads();
        sa_load<T, DP>(sk, g.k, g.ldk, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        sa_load<T, DP>(sv, g.v, g.ldv, (long long)t.k0 + k0, keys, kh * g.head_dim, g.head_dim);
        __syncthreads();
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
        __syncthreads();
        sa_mul<DP>(ss, sk, ty, tx, a, b, acc);
    }
    const float scale[4] = {g.scale, g.scale, g.scale, g.scale};
    sa_store<T, DP>(g.dq, g.lddq, (long long)t.q0 + t.first, rows, h * g.head_dim, g.head_dim, ty, tx, acc, scale);
}

template <int DP>
constexpr int sa_smem(int tiles, int weights) { return (tiles * SA_B * sa_pitch<DP>() + weights * SA_B * SA_PP) * 4; }

template <typename K>
int simt_launch(K kernel, long long grid, int smem, const AttnArgs& g, cudaStream_t s) {
    if (grid > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return ISO_ERR_CUDA;
    TRAIN_LAUNCH((kernel<<<(unsigned)grid, SA_TPB, smem, s>>>(g)));
    return ISO_OK;
}
template <typename T, int DP>
int simt_forward(const AttnArgs& g, cudaStream_t s) {
    return simt_launch(k_simt_attn<T, DP>, attn_tiles(g.q_rows, g.n_seqs, SA_B) * g.heads, sa_smem<DP>(3, 1), g, s);
}
template <typename T, int DP>
int simt_backward(const AttnArgs& g, cudaStream_t s) {
    ISO_TRY(simt_launch(k_simt_grad_kv<T, DP>, attn_tiles(g.k_rows, g.n_seqs, SA_B) * (g.heads / g.group), sa_smem<DP>(4, 2), g, s));
    return simt_launch(k_simt_grad_q<T, DP>, attn_tiles(g.q_rows, g.n_seqs, SA_B) * g.heads, sa_smem<DP>(4, 1), g, s);
}
template <typename F>
int by_kind(int32_t dtype, int dim, F&& f) {
    using B = __nv_bfloat16;
    if (dtype == ISO_BF16) return dim <= 64 ? f((B*)nullptr, std::integral_constant<int, 64>{}) : f((B*)nullptr, std::integral_constant<int, 128>{});
    return dim <= 64 ? f((float*)nullptr, std::integral_constant<int, 64>{}) : f((float*)nullptr, std::integral_constant<int, 128>{});
}

int check_cfg(const iso_attn_cfg* c) {
    if (!c || c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads || c->head_dim < 1) return ISO_ERR_ARG;
    if ((c->causal != 0 && c->causal != 1) || c->window < 0 || (c->window && !c->causal)) return ISO_ERR_ARG;
    if (!(c->scale > 0.0f) || !std::isfinite(c->scale) || c->n_seqs < 0) return ISO_ERR_ARG;
    if ((c->n_seqs > 0) != (c->q_ends != nullptr) || (c->k_ends && !c->q_ends)) return ISO_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(c->q_ends) | reinterpret_cast<uintptr_t>(c->k_ends)) & 3u) return ISO_ERR_ALIGN;
    if (c->head_dim > ISO_ATTN_MAX_DIM) return ISO_ERR_UNSUPPORTED;
    return ISO_OK;
}
constexpr int64_t ATTN_ROWS_LIMIT = 1 << 30;        // a tile's last row and a tile count stay below 2^31
int check_heads(const iso_mat* m, int64_t heads, const iso_attn_cfg* c) {
    ISO_TRY(check_mat(m));
    if (m->cols != heads * c->head_dim) return ISO_ERR_SHAPE;
    if (m->rows > ATTN_ROWS_LIMIT) return ISO_ERR_UNSUPPORTED;
    return ISO_OK;
}
int check_qk(const iso_mat* q, const iso_mat* k, const iso_attn_cfg* c) {
    ISO_TRY(check_cfg(c));
    ISO_TRY(check_heads(q, c->heads, c));
    ISO_TRY(check_heads(k, c->kv_heads, c));
    if (c->q_ends && !c->k_ends && k->rows != q->rows) return ISO_ERR_SHAPE;
    if (k->dtype != q->dtype) return ISO_ERR_DTYPE;
    return ISO_OK;
}
int check_like(const iso_mat* m, const iso_mat* like) {
    ISO_TRY(check_mat(m));
    if (m->rows != like->rows || m->cols != like->cols) return ISO_ERR_SHAPE;
    return m->dtype == like->dtype ? ISO_OK : ISO_ERR_DTYPE;
}
Bytes2D ends_bytes(const int32_t* p, int n) {
    const uint64_t b = p ? ((uint64_t)n + 1) * 4 : 0;
    return {reinterpret_cast<uintptr_t>(p), 1, b, b};
}
Bytes2D floats(const float* p, uint64_t n) { return {reinterpret_cast<uintptr_t>(p), 1, 4 * n, 4 * n}; }
// no output over an input or another output
template <int I, int O>
bool overlap(const Bytes2D (&in)[I], const Bytes2D (&out)[O]) {
    for (int o = 0; o < O; ++o) {
        for (int i = 0; i < I; ++i)
            if (share_bytes(out[o], in[i])) return true;
        for (int p = 0; p < o; ++p)
            if (share_bytes(out[o], out[p])) return true;
    }
    return false;
}

AttnArgs attn_args(const iso_mat* q, const iso_mat* k, const iso_mat* v, const iso_mat* out, const float* lse,
                   const iso_attn_cfg* c, int32_t* status) {
    AttnArgs g{};
    g.q = q->data; g.k = k->data; g.v = v->data; g.out = out->data;
    g.ldq = q->ld; g.ldk = k->ld; g.ldv = v->ld; g.ldo = out->ld;
    g.lse = const_cast<float*>(lse);
    g.q_rows = (int)q->rows;
    g.k_rows = (int)k->rows;
    g.heads = c->heads;
    g.group = c->heads / c->kv_heads;
    g.head_dim = c->head_dim;
    g.causal = c->causal;
    g.window = std::min<int64_t>(c->window, 1LL << 40);
    g.scale = c->scale;
    g.n_seqs = c->n_seqs;
    g.q_ends = c->q_ends;
    g.k_ends = c->k_ends ? c->k_ends : c->q_ends;
    g.status = status;
    return g;
}
size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_attn_workspace_size(const iso_mat* q, const iso_mat* k, const iso_attn_cfg* cfg, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_qk(q, k, cfg));
    *bytes = 256;
    return ISO_OK;
}

int32_t iso_attn(const iso_mat* q, const iso_mat* k, const iso_mat* v, const iso_attn_cfg* cfg, const iso_mat* out,
                 float* lse, void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    ISO_TRY(check_qk(q, k, cfg));
    ISO_TRY(check_like(v, k));
    ISO_TRY(check_like(out, q));
    if (q->rows && !lse) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return ISO_ERR_ALIGN;
    const Bytes2D in[5] = {bytes_of(q), bytes_of(k), bytes_of(v), ends_bytes(cfg->q_ends, cfg->n_seqs), ends_bytes(cfg->k_ends, cfg->n_seqs)};
    const Bytes2D outs[2] = {bytes_of(out), floats(lse, (uint64_t)q->rows * cfg->heads)};
    if (overlap(in, outs)) return ISO_ERR_ARG;
    if (!workspace || ws_bytes < 256 || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (q->rows == 0) return ISO_OK;
    const AttnArgs g = attn_args(q, k, v, out, lse, cfg, status);
    return by_kind(q->dtype, cfg->head_dim, [&](auto* t, auto dp) -> int {
        return simt_forward<std::remove_pointer_t<decltype(t)>, decltype(dp)::value>(g, s);
    });
}

int32_t iso_attn_grad_workspace_size(const iso_mat* q, const iso_mat* k, const iso_attn_cfg* cfg, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_qk(q, k, cfg));
    *bytes = round256((size_t)q->rows * cfg->heads * 4) + 256;
    return ISO_OK;
}

int32_t iso_attn_grad(const iso_mat* dout, const iso_mat* q, const iso_mat* k, const iso_mat* v, const iso_mat* out,
                      const float* lse, const iso_attn_cfg* cfg, const iso_mat* dq, const iso_mat* dk,
                      const iso_mat* dv, void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    ISO_TRY(check_qk(q, k, cfg));
    ISO_TRY(check_like(v, k));
    for (const iso_mat* m : {out, dout, dq}) ISO_TRY(check_like(m, q));
    for (const iso_mat* m : {dk, dv}) ISO_TRY(check_like(m, k));
    if (q->rows && !lse) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return ISO_ERR_ALIGN;
    const Bytes2D in[8] = {bytes_of(q), bytes_of(k), bytes_of(v), bytes_of(out), bytes_of(dout),
                           floats(lse, (uint64_t)q->rows * cfg->heads), ends_bytes(cfg->q_ends, cfg->n_seqs),
                           ends_bytes(cfg->k_ends, cfg->n_seqs)};
    const Bytes2D outs[3] = {bytes_of(dq), bytes_of(dk), bytes_of(dv)};
    if (overlap(in, outs)) return ISO_ERR_ARG;
    size_t need = 0;
    ISO_TRY(iso_attn_grad_workspace_size(q, k, cfg, &need));
    if (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (q->rows == 0 && k->rows == 0) return ISO_OK;
    AttnArgs g = attn_args(q, k, v, out, lse, cfg, status);
    g.dout = dout->data;
    g.lddo = dout->ld;
    g.dq = dq->data; g.dk = dk->data; g.dv = dv->data;
    g.lddq = dq->ld; g.lddk = dk->ld; g.lddv = dv->ld;
    g.delta = static_cast<float*>(workspace);
    return by_kind(q->dtype, cfg->head_dim, [&](auto* t, auto dp) -> int {
        using T = std::remove_pointer_t<decltype(t)>;
        if (q->rows) {
            const long long warps = (long long)q->rows * cfg->heads;
            if ((warps + 7) / 8 > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
            TRAIN_LAUNCH((k_attn_delta<T><<<(unsigned)((warps + 7) / 8), 256, 0, s>>>(g)));
        }
        return simt_backward<T, decltype(dp)::value>(g, s);
    });
}

}  // extern "C"
