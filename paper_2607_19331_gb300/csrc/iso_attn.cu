// iso_attn.cu -- attention and its gradients: entry points, and the kernels on
// the CUDA cores.
//
// Forward: one pass over the keys with the running maximum m and sum l of the
// softmax: O <- O e^(m - m') + e^(S - m') V.  Backward: the weights again from
// lse, P = e^(S - lse), and no atomics: some CTAs own a tile of keys and go over the
// queries (of all query heads of its key head), others own a tile of queries and go
// over the keys; S and dP are formed in both (seven
// products instead of five), and every sum has a fixed order.
//
// The CUDA-core kernels (tiles in iso_attn_simt.cuh) take any type, head
// dimension, stride and alignment, in binary32 throughout.
#include "iso_attn.cuh"
#include "iso_attn_simt.cuh"
#include "iso_attn_tc.cuh"
#include "iso_tc.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace iso {
namespace {

// Zeros in the rows of up to three outputs, and the columns of lse, that belong to
// no sequence: before the first one and behind the last.
struct Rest {
    void* at[3];
    long long ld[3];
    int32_t rows[3], cols[3];            // cols: bytes of a row / 2
    const int32_t* ends[3];
    float* lse;
    int32_t n_seqs, heads;
};
__global__ void __launch_bounds__(256) k_zero_rest(const __grid_constant__ Rest z) {
    auto each = [&](int m, auto f) {
        const int first = min(max(z.ends[m][0], 0), z.rows[m]), last = max(first, min(max(z.ends[m][z.n_seqs], 0), z.rows[m]));
        for (int r = blockIdx.x; r < first + z.rows[m] - last; r += gridDim.x) f(r < first ? r : last + r - first);
    };
    for (int m = 0; m < 3; ++m) {
        if (!z.at[m]) continue;
        each(m, [&](int row) {
            uint16_t* p = static_cast<uint16_t*>(z.at[m]) + row * z.ld[m];
            for (int c = threadIdx.x; c < z.cols[m]; c += blockDim.x) p[c] = 0;
            if (m == 0 && z.lse)
                for (int h = threadIdx.x; h < z.heads; h += blockDim.x) z.lse[(long long)h * z.rows[0] + row] = 0.0f;
        });
    }
}
int zero_rest(const AttnArgs& g, const iso_mat* a, const iso_mat* b, const iso_mat* c, float* lse, cudaStream_t s) {
    if (g.n_seqs == 0) return ISO_OK;
    Rest z{};
    const iso_mat* mats[3] = {a, b, c};
    for (int m = 0; m < 3; ++m) {
        if (!mats[m] || mats[m]->rows == 0) continue;
        const int halves = elem_size(mats[m]->dtype) / 2;
        z.at[m] = mats[m]->data;
        z.ld[m] = mats[m]->ld * halves;
        z.rows[m] = (int)mats[m]->rows;
        z.cols[m] = (int)(mats[m]->cols * halves);
        z.ends[m] = m == 0 ? g.q_ends : g.k_ends;
    }
    z.lse = lse;
    z.n_seqs = g.n_seqs;
    z.heads = g.heads;
    TRAIN_LAUNCH((k_zero_rest<<<(unsigned)std::min(train_sms(), 152), 256, 0, s>>>(z)));
    return ISO_OK;
}

template <typename T, int DP>
__global__ void __launch_bounds__(SA_TPB) k_simt_attn(AttnArgs g) {
    extern __shared__ __align__(16) float sa_smem_[];
    AttnTile t;
    if (attn_find_tile(g, blockIdx.x / g.heads, SA_B, false, t))
        simt_attn<T, DP, T>(g, t, blockIdx.x % g.heads, 0, t.nk, static_cast<T*>(const_cast<void*>(g.out)), g.ldo, g.lse, sa_smem_);
}
// one launch for both: the keys' CTAs first
template <typename T, int DP>
__global__ void __launch_bounds__(SA_TPB) k_simt_grad(AttnArgs g, int kv_items) {
    extern __shared__ __align__(16) float sa_smem_[];
    AttnTile t;
    if ((int)blockIdx.x < kv_items) {
        const int kv_heads = g.heads / g.group, kh = blockIdx.x % kv_heads;
        if (attn_find_tile(g, blockIdx.x / kv_heads, SA_B, true, t))
            simt_grad_kv<T, DP, T>(g, t, kh, kh * g.group, (kh + 1) * g.group, static_cast<T*>(g.dk), g.lddk, static_cast<T*>(g.dv),
                                   g.lddv, sa_smem_);
    } else {
        const int i = (int)blockIdx.x - kv_items;
        if (attn_find_tile(g, i / g.heads, SA_B, false, t)) simt_grad_q<T, DP>(g, t, i % g.heads, sa_smem_);
    }
}

// delta[h][i] = sum_d dout_id out_id, heads that are whole 16-byte words at such
// boundaries: a word of both a lane, 16 lanes a row and head, DELTA_EACH of them in
// flight (8269 rows of 12 heads: 13.4 us, a lane a channel 18.4)
constexpr int DELTA_EACH = 4;
__global__ void __launch_bounds__(256) k_attn_delta_words(AttnArgs g) {
    const long long n = (long long)g.q_rows * g.heads, group = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 4;
    const int lane = threadIdx.x & 15, c = lane * 8;
    const bool in = c < g.head_dim;
    uint4 o[DELTA_EACH], d[DELTA_EACH];
#pragma unroll
    for (int j = 0; j < DELTA_EACH; ++j) {
        const long long i = group * DELTA_EACH + j, row = i / g.heads, h = i - row * g.heads;
        o[j] = d[j] = make_uint4(0u, 0u, 0u, 0u);
        if (i < n && in) {
            o[j] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(g.out) + row * g.ldo + h * g.head_dim + c));
            d[j] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(g.dout) + row * g.lddo + h * g.head_dim + c);
        }
    }
#pragma unroll
    for (int j = 0; j < DELTA_EACH; ++j) {
        const long long i = group * DELTA_EACH + j, row = i / g.heads, h = i - row * g.heads;
        const uint32_t a[4] = {o[j].x, o[j].y, o[j].z, o[j].w}, b[4] = {d[j].x, d[j].y, d[j].z, d[j].w};
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x, y, u, w;
            bf16x2_to_f32(a[k], x, y);
            bf16x2_to_f32(b[k], u, w);
            s = fmaf(x, u, s);
            s = fmaf(y, w, s);
        }
#pragma unroll
        for (int k = 8; k; k >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
        if (lane == 0 && i < n) g.delta[h * g.q_rows + row] = s;
    }
}

// The same of any head: a warp per row and head
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

template <typename T, int DP>
int simt_forward(const AttnArgs& g, cudaStream_t s) {
    const long long grid = attn_tiles(g.q_rows, g.n_seqs, SA_B) * g.heads;
    if (grid > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> done{0};
    ISO_TRY(allow_smem(k_simt_attn<T, DP>, sa_smem<DP>(3, 1), done));
    TRAIN_LAUNCH((k_simt_attn<T, DP><<<(unsigned)grid, SA_TPB, sa_smem<DP>(3, 1), s>>>(g)));
    return ISO_OK;
}
template <typename T, int DP>
int simt_backward(const AttnArgs& g, cudaStream_t s) {
    const long long kv = attn_tiles(g.k_rows, g.n_seqs, SA_B) * (g.heads / g.group), q = attn_tiles(g.q_rows, g.n_seqs, SA_B) * g.heads;
    if (kv + q > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> done{0};
    ISO_TRY(allow_smem(k_simt_grad<T, DP>, sa_smem<DP>(4, 2), done));
    TRAIN_LAUNCH((k_simt_grad<T, DP><<<(unsigned)(kv + q), SA_TPB, sa_smem<DP>(4, 2), s>>>(g, (int)kv)));
    return ISO_OK;
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
    if ((c->zero_rest != 0 && c->zero_rest != 1) || c->reserved != 0) return ISO_ERR_ARG;
    if (!(c->scale > 0.0f) || !std::isfinite(c->scale * tc::LOG2E) || c->n_seqs < 0) return ISO_ERR_ARG;
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

// what tensor copies can take: heads and rows on 16-byte boundaries
bool copies_take(const iso_mat* m) {
    return (reinterpret_cast<uintptr_t>(m->data) & 15u) == 0 && (m->rows == 1 || (m->ld * 2) % 16 == 0);
}
template <typename... M>
bool on_tensor_cores(const iso_attn_cfg* c, const M*... m) {
    return c->head_dim % 8 == 0 && ((m->dtype == ISO_BF16) && ...) && (copies_take(m) && ...) && ((m->rows > 0) && ...);
}

constexpr uint64_t ATTN_WAIT_NS = 2000000000;      // a wait gives up after this long, unless told otherwise
std::atomic<uint64_t> g_attn_wait_ns{ATTN_WAIT_NS};

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                       q == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<EncodeTiled>(p)
                   : nullptr;
    }();
    return fn;
}

}  // namespace

uint64_t attn_wait_ns() { return g_attn_wait_ns.load(std::memory_order_relaxed); }

int tc::head_map(CUtensorMap* map, const void* base, long long rows, int heads, int head_dim, long long ld) {
    EncodeTiled fn = encode_tiled();
    if (!fn) return ISO_ERR_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)rows};
    // (of a single row any stride does)
    const cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)(rows == 1 ? (long long)heads * head_dim : ld) * 2};
    const cuuint32_t box[3] = {(cuuint32_t)BOX, 1, (cuuint32_t)ROWS};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? ISO_OK
               : ISO_ERR_CUDA;
}

}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_attn_workspace_size(const iso_mat* q, const iso_mat* k, const iso_attn_cfg* cfg, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_qk(q, k, cfg));
    *bytes = round256(attn_plan(q->rows, k->rows, *cfg).bytes) + 256;
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
    size_t need = 0;
    ISO_TRY(iso_attn_workspace_size(q, k, cfg, &need));
    if (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (q->rows == 0) return ISO_OK;
    const AttnArgs g = attn_args(q, k, v, out, lse, cfg, status);
    if (cfg->zero_rest) ISO_TRY(zero_rest(g, out, nullptr, nullptr, lse, s));
    if (on_tensor_cores(cfg, q, k, v)) return attn_tc(g, attn_plan(q->rows, k->rows, *cfg), static_cast<float*>(workspace), s);
    return by_kind(q->dtype, cfg->head_dim, [&](auto* t, auto dp) -> int {
        return simt_forward<std::remove_pointer_t<decltype(t)>, decltype(dp)::value>(g, s);
    });
}

int32_t iso_attn_grad_workspace_size(const iso_mat* q, const iso_mat* k, const iso_attn_cfg* cfg, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_qk(q, k, cfg));
    *bytes = round256((size_t)q->rows * cfg->heads * 4) + round256(attn_grad_plan(q->rows, k->rows, *cfg).bytes) + 256;
    return ISO_OK;
}

int64_t iso_attn_wait_ns(int64_t ns) {
    return (int64_t)(ns < 0 ? g_attn_wait_ns.load(std::memory_order_relaxed)
                            : g_attn_wait_ns.exchange((uint64_t)ns, std::memory_order_relaxed));
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
    if (cfg->zero_rest) ISO_TRY(zero_rest(g, dq, dk, dv, nullptr, s));
    return by_kind(q->dtype, cfg->head_dim, [&](auto* t, auto dp) -> int {
        using T = std::remove_pointer_t<decltype(t)>;
        if (q->rows) {
            const long long warps = (long long)q->rows * cfg->heads;
            if ((warps + 7) / 8 > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
            if (on_tensor_cores(cfg, out, dout)) {
                const long long groups = (warps + DELTA_EACH - 1) / DELTA_EACH;
                TRAIN_LAUNCH((k_attn_delta_words<<<(unsigned)((groups + 15) / 16), 256, 0, s>>>(g)));
            } else {
                TRAIN_LAUNCH((k_attn_delta<T><<<(unsigned)((warps + 7) / 8), 256, 0, s>>>(g)));
            }
        }
        if (on_tensor_cores(cfg, q, k, v, dout))
            return attn_grad_tc(g, attn_grad_plan(q->rows, k->rows, *cfg),
                                reinterpret_cast<float*>(static_cast<char*>(workspace) + round256((size_t)q->rows * cfg->heads * 4)), s);
        return simt_backward<T, decltype(dp)::value>(g, s);
    });
}

}  // extern "C"
