// iso_embed.cu -- the token embedding and its gradient by sorted tokens.
//
// Forward: a gather of table rows, bound by HBM; a warp takes 256 channels of
// one token at a time (16-byte loads).
//
// Gradient: grad[v] = scale * sum of dY[t] over the tokens of id v.
//   k_sort_fill  one cluster of eight CTAs sorts (id, token) by a stable LSD
//                radix sort, digits of up to nine bits, while the other CTAs
//                write the zeros of a gradient that is not accumulated (a
//                vocabulary has far more rows than a batch has tokens, so the
//                zeros are the bulk of the traffic and hide the sort; rows
//                with tokens are written a second time);
//   k_row_sums   sorted tokens in windows of 32: a warp adds the window's dY
//                rows over 256 channels and writes the sum of every run of
//                equal ids that lies inside the window; a run that crosses a
//                window's edge leaves one partial row per window;
//   k_row_join   the runs that cross windows: partials added, row written.
// Sums are binary32 and their order is fixed by the sorted positions: windows
// of 32 in ascending token order, then the window sums, so equal inputs give
// equal bits and a frequent id's sum is a short tree, not one long chain.
#include "iso_train.cuh"

#include <algorithm>
#include <cmath>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace iso {
namespace {

constexpr int EM_TPB = 256;
constexpr int EM_WPB = EM_TPB / 32;

constexpr int SORT_CLUSTER = 8;
constexpr int SORT_TPB = 1024;
constexpr int SORT_WARPS = SORT_TPB / 32;
constexpr int SORT_BITS = 9;
constexpr int SORT_BINS = 1 << SORT_BITS;
constexpr int FILL_CHUNK = 16384;                       // bytes of zeros a warp writes at a time
constexpr int WIN = 32;                                 // sorted tokens per window
constexpr int JOIN_TPB = 512;
constexpr int JOIN_COLS = 128;

struct Ids {
    const void* p;
    long long n;
    long long pad_id;
    long long rows;     // table rows
    int i64;
};
__device__ __forceinline__ long long load_id(const Ids& ids, long long t) {
    return ids.i64 ? static_cast<const long long*>(ids.p)[t] : (long long)static_cast<const int*>(ids.p)[t];
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(EM_TPB) k_embed(const T* table, long long ldt, Ids ids, float scale, O* out,
                                                  long long ldo, int cols, int segs, int32_t* status) {
    const int lane = threadIdx.x & 31;
    const long long items = ids.n * segs, warps = (long long)gridDim.x * EM_WPB;
    for (long long i = (long long)blockIdx.x * EM_WPB + (threadIdx.x >> 5); i < items; i += warps) {
        const long long t = i / segs;
        const int c = (int)(i - t * segs) * TRAIN_SEG + lane * 8;
        const long long id = load_id(ids, t);
        float v[8] = {};
        if (id == ids.pad_id) {
        } else if (id >= 0 && id < ids.rows) {
            load8<VEC>(table + id * ldt, c, cols, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= scale;
        } else if (status && lane == 0) {
            *status = ISO_ERR_INDEX;
        }
        store8<VEC>(out + t * ldo, c, cols, v);
    }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
struct FillArgs {
    char* base;             // NULL: nothing to fill
    long long rows;         // runs of `width` bytes, `stride` apart
    long long width, stride;
};

// zeros over len bytes from p (both multiples of two) by one warp
__device__ __forceinline__ void warp_zero(char* p, long long len, int lane) {
    const long long head = min(len, (long long)((16 - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u));
    for (long long i = 2 * lane; i < head; i += 64) *reinterpret_cast<uint16_t*>(p + i) = 0;
    p += head;
    len -= head;
    const long long vecs = len / 16;
    for (long long i = lane; i < vecs; i += 32) reinterpret_cast<uint4*>(p)[i] = make_uint4(0u, 0u, 0u, 0u);
    for (long long i = vecs * 16 + 2 * lane; i < len; i += 64) *reinterpret_cast<uint16_t*>(p + i) = 0;
}

__device__ void fill_zeros(const FillArgs& f, long long warp, long long warps, int lane) {
    const long long per_row = (f.width + FILL_CHUNK - 1) / FILL_CHUNK;
    for (long long i = warp; i < f.rows * per_row; i += warps) {
        const long long r = i / per_row, off = (i - r * per_row) * FILL_CHUNK;
        warp_zero(f.base + r * f.stride + off, min((long long)FILL_CHUNK, f.width - off), lane);
    }
}

struct SortArgs {
    Ids ids;
    uint2* buf[2];          // {id, token}; the sorted list ends in buf[0]; padding and bad ids as id = rows, last
    int passes, bits;
    int32_t* status;
    uint32_t* n_joins;      // cleared for k_row_sums
};

__device__ __forceinline__ uint2 sort_item(const SortArgs& a, const uint2* src, long long t, bool& bad) {
    if (src) return src[t];
    const long long id = load_id(a.ids, t);
    const bool pad = id == a.ids.pad_id, in = id >= 0 && id < a.ids.rows;
    bad |= !pad && !in;
    return make_uint2(!pad && in ? (uint32_t)id : (uint32_t)a.ids.rows, (uint32_t)t);
}

__global__ void __cluster_dims__(SORT_CLUSTER, 1, 1) __launch_bounds__(SORT_TPB)
k_sort_fill(SortArgs a, FillArgs f) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x >= SORT_CLUSTER) {
        fill_zeros(f, (long long)(blockIdx.x - SORT_CLUSTER) * SORT_WARPS + warp,
                   (long long)(gridDim.x - SORT_CLUSTER) * SORT_WARPS, lane);
        return;
    }
    extern __shared__ uint32_t sort_smem[];
    uint32_t* const cnt = sort_smem;                                  // [warp][bin]
    uint32_t* const tot = cnt + SORT_WARPS * SORT_BINS;               // [bin]: this CTA's items
    uint32_t* const scan = tot + SORT_BINS;                           // [warp sums]
    int* const bad_flag = reinterpret_cast<int*>(scan + 32);
    cg::cluster_group cluster = cg::this_cluster();
    const int me = (int)cluster.block_rank();
    const uint32_t lt = (1u << lane) - 1u;
    // every warp owns a contiguous range of positions, in order, so that ranks
    // counted range by range are stable
    const long long n = a.ids.n;
    const long long per = ((n + SORT_CLUSTER * SORT_WARPS - 1) / (SORT_CLUSTER * SORT_WARPS) + 31) / 32 * 32;
    const long long t0 = min(n, ((long long)me * SORT_WARPS + warp) * per), t1 = min(n, t0 + per);
    if (threadIdx.x == 0) *bad_flag = 0;
    __syncthreads();
    bool bad = false;
    for (int p = 0; p < a.passes; ++p) {
        const uint2* src = p == 0 ? nullptr : a.buf[(a.passes - p) & 1];
        uint2* dst = a.buf[(a.passes - 1 - p) & 1];
        const int shift = p * a.bits;
        const uint32_t mask = (1u << a.bits) - 1u;
        for (int i = threadIdx.x; i < SORT_WARPS * SORT_BINS; i += SORT_TPB) cnt[i] = 0;
        __syncthreads();
        uint32_t* const mine = cnt + warp * SORT_BINS;
        for (long long b = t0; b < t1; b += 32) {
            const bool on = b + lane < t1;
            const uint32_t active = __ballot_sync(0xFFFFFFFFu, on);
            if (on) {
                const uint32_t d = (sort_item(a, src, b + lane, bad).x >> shift) & mask;
                const uint32_t same = __match_any_sync(active, d);
                if ((same & lt) == 0) mine[d] += __popc(same);
            }
            __syncwarp();
        }
        if (bad) *bad_flag = 1;
        __syncthreads();
        // bins: prefix over this CTA's warps, the CTA's total
        if (threadIdx.x < SORT_BINS) {
            uint32_t s = 0;
            for (int w = 0; w < SORT_WARPS; ++w) {
                const uint32_t v = cnt[w * SORT_BINS + threadIdx.x];
                cnt[w * SORT_BINS + threadIdx.x] = s;
                s += v;
            }
            tot[threadIdx.x] = s;
        }
        cluster.sync();
        // start of each bin for this CTA: earlier bins of all CTAs, earlier CTAs of this bin
        uint32_t all = 0, before = 0;
        if (threadIdx.x < SORT_BINS) {
            for (int c = 0; c < SORT_CLUSTER; ++c) {
                const uint32_t v = cluster.map_shared_rank(tot, c)[threadIdx.x];
                all += v;
                if (c < me) before += v;
            }
        }
        uint32_t inc = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) scan[warp] = inc;
        __syncthreads();
        if (threadIdx.x < SORT_BINS) {
            uint32_t base = before + inc - all;
            for (int w = 0; w < warp; ++w) base += scan[w];
            for (int w = 0; w < SORT_WARPS; ++w) cnt[w * SORT_BINS + threadIdx.x] += base;
        }
        __syncthreads();
        for (long long b = t0; b < t1; b += 32) {
            const bool on = b + lane < t1;
            const uint32_t active = __ballot_sync(0xFFFFFFFFu, on);
            if (on) {
                const uint2 it = sort_item(a, src, b + lane, bad);
                const uint32_t d = (it.x >> shift) & mask;
                const uint32_t same = __match_any_sync(active, d);
                const uint32_t at = mine[d];
                __syncwarp(active);
                if ((same & lt) == 0) mine[d] = at + __popc(same);
                dst[at + __popc(same & lt)] = it;
            }
            __syncwarp();
        }
        if (p == 0 && me == 0 && threadIdx.x == 0) {
            int any = 0;
            for (int c = 0; c < SORT_CLUSTER; ++c) any |= *cluster.map_shared_rank(bad_flag, c);
            if (a.status) *a.status = any ? (int32_t)ISO_ERR_INDEX : (int32_t)ISO_OK;
            *a.n_joins = 0;
        }
        cluster.sync();   // dst is complete; no CTA still reads another's shared memory
    }
}

struct RowArgs {
    const uint2* sorted;
    long long n;
    uint32_t rows;          // table rows: the id of padding
    float scale;
    int cols, segs, accumulate;
    float* part;            // [window][2][cols]: the run that enters the window, the run that leaves it
    long long ld_part;
    uint32_t* joins;        // windows whose last run starts there and goes on
    uint32_t* n_joins;
};

template <typename O, bool VEC>
__device__ __forceinline__ void write_row(O* row, int c, int cols, float (&v)[8], float scale, int accumulate) {
    if (c >= cols) return;
    if (accumulate) {
        float old[8];
        load8<VEC>(row, c, cols, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = old[j] + v[j] * scale;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= scale;
    }
    store8<VEC>(row, c, cols, v);
}

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(EM_TPB) k_row_sums(const T* dy, long long ldd, O* grad, long long ldg, RowArgs a) {
    const int lane = threadIdx.x & 31;
    const long long wins = (a.n + WIN - 1) / WIN, items = wins * a.segs, warps = (long long)gridDim.x * EM_WPB;
    for (long long i = (long long)blockIdx.x * EM_WPB + (threadIdx.x >> 5); i < items; i += warps) {
        const long long w = i / a.segs;
        const int seg = (int)(i - w * a.segs), c = seg * TRAIN_SEG + lane * 8;
        const long long p0 = w * WIN;
        const uint2 it = p0 + lane < a.n ? a.sorted[p0 + lane] : make_uint2(a.rows, 0u);
        const uint32_t prev = p0 > 0 ? a.sorted[p0 - 1].x : 0xFFFFFFFFu;
        const uint32_t next = p0 + WIN < a.n ? a.sorted[p0 + WIN].x : 0xFFFFFFFFu;
        float acc[8] = {};
        bool enters = __shfl_sync(0xFFFFFFFFu, it.x, 0) == prev;
        constexpr int UN = 8;
#pragma unroll 1
        for (int b = 0; b < WIN; b += UN) {
            float v[UN][8];
#pragma unroll
            for (int j = 0; j < UN; ++j) {
                const uint32_t id = __shfl_sync(0xFFFFFFFFu, it.x, b + j), pos = __shfl_sync(0xFFFFFFFFu, it.y, b + j);
                if (id < a.rows) load8<VEC>(dy + (long long)pos * ldd, c, a.cols, v[j]);
            }
#pragma unroll
            for (int j = 0; j < UN; ++j) {
                const uint32_t id = __shfl_sync(0xFFFFFFFFu, it.x, b + j);
                if (id >= a.rows) break;
                const uint32_t nx = __shfl_sync(0xFFFFFFFFu, it.x, (b + j + 1) & 31);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] += v[j][k];
                const bool last = b + j == WIN - 1;
                const bool leaves = last && next == id;
                if (!last && nx == id) continue;
                if (!enters && !leaves) {
                    write_row<O, VEC>(grad + (long long)id * ldg, c, a.cols, acc, a.scale, a.accumulate);
                } else if (c < a.cols) {
                    float* part = a.part + (w * 2 + (enters ? 0 : 1)) * a.ld_part;
                    store8<true>(part, c, (int)a.ld_part, acc);
                }
                if (!enters && leaves && seg == 0 && lane == 0) a.joins[atomicAdd(a.n_joins, 1u)] = (uint32_t)w;
                enters = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = 0.0f;
            }
        }
    }
}

template <typename O, bool VEC>
__global__ void __launch_bounds__(JOIN_TPB) k_row_join(O* grad, long long ldg, RowArgs a) {
    __shared__ float4 sums[JOIN_TPB / 32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int WARPS = JOIN_TPB / 32;
    const int slices = (a.cols + JOIN_COLS - 1) / JOIN_COLS;
    const long long items = (long long)*a.n_joins * slices, wins = (a.n + WIN - 1) / WIN;
    for (long long i = blockIdx.x; i < items; i += gridDim.x) {
        const long long e = i / slices, w = a.joins[e];
        const int c = (int)(i - e * slices) * JOIN_COLS + lane * 4;
        const uint32_t id = a.sorted[w * WIN + WIN - 1].x;
        // windows w + 1 .. w + k whose first token continues the run
        long long k = 0;
        for (;;) {
            const long long q = w + 1 + k + threadIdx.x;
            const int got = __syncthreads_count(q < wins && a.sorted[q * WIN].x == id);
            k += got;
            if (got < JOIN_TPB) break;
        }
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        const bool on = c < a.cols;                       // part rows are padded to a multiple of 8
        // part row of step q: the leaving run of w, then the entering runs of w + 1 ..
        if (on) {
#pragma unroll 4
            for (long long q = warp; q <= k; q += WARPS) {
                const float4 v = *reinterpret_cast<const float4*>(a.part + ((w + q) * 2 + (q == 0 ? 1 : 0)) * a.ld_part + c);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        }
        sums[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && on) {
            for (int q = 1; q < WARPS; ++q) {
                const float4 v = sums[q][lane];
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            const float r[4] = {s.x, s.y, s.z, s.w};
            O* row = grad + (long long)id * ldg;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < a.cols) from_f32(a.accumulate ? to_f32(row[c + j]) + r[j] * a.scale : r[j] * a.scale, row[c + j]);
        }
        __syncthreads();
    }
}

int check_ids(const void* ids, int32_t i64, int64_t n) {
    if (i64 != 0 && i64 != 1) return ISO_ERR_ARG;
    if (n < 0) return ISO_ERR_SHAPE;
    if (n > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    if (n == 0) return ISO_OK;
    if (!ids) return ISO_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ids) % (i64 ? 8 : 4)) return ISO_ERR_ALIGN;
    return ISO_OK;
}
Bytes2D ids_bytes(const void* ids, int32_t i64, int64_t n) {
    return {reinterpret_cast<uintptr_t>(ids), n > 0 ? 1u : 0u, (uint64_t)n * (i64 ? 8 : 4), (uint64_t)n * (i64 ? 8 : 4)};
}

// workspace: header (join count), the two sort buffers, the join list, the partial rows
struct GradLayout {
    size_t buf0, buf1, joins, part, end;
    long long ld_part;
};
GradLayout grad_layout(int64_t n, int64_t cols) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    const size_t wins = (size_t)((n + WIN - 1) / WIN);
    GradLayout L;
    L.ld_part = (cols + 7) / 8 * 8;
    L.buf0 = 256;
    L.buf1 = L.buf0 + up((size_t)n * sizeof(uint2));
    L.joins = L.buf1 + up((size_t)n * sizeof(uint2));
    L.part = L.joins + up(wins * sizeof(uint32_t));
    L.end = L.part + up(wins * 2 * (size_t)L.ld_part * sizeof(float));
    return L;
}

template <typename F>
int dispatch2(int32_t ta, int32_t tb, bool vec, F&& f) {
    using B = __nv_bfloat16;
    auto with = [&](auto* a, auto* b) { return vec ? f(a, b, std::true_type{}) : f(a, b, std::false_type{}); };
    if (ta == ISO_BF16) return tb == ISO_BF16 ? with((B*)nullptr, (B*)nullptr) : with((B*)nullptr, (float*)nullptr);
    return tb == ISO_BF16 ? with((float*)nullptr, (B*)nullptr) : with((float*)nullptr, (float*)nullptr);
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_embed(const iso_mat* table, const void* ids, int32_t ids_i64, int64_t n, int64_t pad_id, float scale,
                  const iso_mat* out, int32_t* status, void* stream) {
    ISO_TRY(check_mat(table));
    ISO_TRY(check_mat(out));
    ISO_TRY(check_ids(ids, ids_i64, n));
    if (out->rows != n || out->cols != table->cols) return ISO_ERR_SHAPE;
    if (!std::isfinite(scale)) return ISO_ERR_ARG;
    if (share_bytes(bytes_of(out), bytes_of(table)) || share_bytes(bytes_of(out), ids_bytes(ids, ids_i64, n)))
        return ISO_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (n == 0 || out->cols == 0) return ISO_OK;
    const Ids id{ids, (long long)n, (long long)pad_id, (long long)table->rows, ids_i64};
    const int segs = (int)((out->cols + TRAIN_SEG - 1) / TRAIN_SEG);
    const int grid = (int)std::max(1LL, std::min(((long long)n * segs + EM_WPB - 1) / EM_WPB, (long long)train_sms() * 8));
    return dispatch2(table->dtype, out->dtype, rows_aligned(table) && rows_aligned(out), [&](auto* tp, auto* op, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        TRAIN_LAUNCH((k_embed<T, O, decltype(v)::value><<<grid, EM_TPB, 0, s>>>(
            static_cast<const T*>(table->data), table->ld, id, scale, static_cast<O*>(out->data), out->ld,
            (int)out->cols, segs, status)));
        return ISO_OK;
    });
}

int32_t iso_embed_grad_workspace_size(int64_t n, int64_t cols, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    if (n < 0 || cols < 0) return ISO_ERR_SHAPE;
    if (n > EXTENT_LIMIT || cols > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    *bytes = grad_layout(n, cols).end;
    return ISO_OK;
}

int32_t iso_embed_grad(const iso_mat* dY, const void* ids, int32_t ids_i64, int64_t pad_id, float scale,
                       const iso_mat* grad, int32_t accumulate, void* workspace, size_t ws_bytes, int32_t* status,
                       void* stream) {
    ISO_TRY(check_mat(dY));
    ISO_TRY(check_mat(grad));
    const int64_t n = dY->rows;
    ISO_TRY(check_ids(ids, ids_i64, n));
    if (grad->cols != dY->cols) return ISO_ERR_SHAPE;
    if (!std::isfinite(scale)) return ISO_ERR_ARG;
    if (accumulate != 0 && accumulate != 1) return ISO_ERR_ARG;
    if (share_bytes(bytes_of(grad), bytes_of(dY)) || share_bytes(bytes_of(grad), ids_bytes(ids, ids_i64, n)))
        return ISO_ERR_ARG;
    const GradLayout L = grad_layout(n, grad->cols);
    if (!workspace || ws_bytes < L.end || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);

    SortArgs sa;
    sa.ids = {ids, (long long)n, (long long)pad_id, (long long)grad->rows, ids_i64};
    sa.buf[0] = reinterpret_cast<uint2*>(ws + L.buf0);
    sa.buf[1] = reinterpret_cast<uint2*>(ws + L.buf1);
    int bits = 1;                                            // ids 0 .. rows, rows marking padding
    while (bits < 31 && ((int64_t)grad->rows >> bits)) ++bits;
    sa.passes = (bits + SORT_BITS - 1) / SORT_BITS;
    sa.bits = (bits + sa.passes - 1) / sa.passes;
    sa.status = status;
    sa.n_joins = reinterpret_cast<uint32_t*>(ws);
    const int es = elem_size(grad->dtype);
    FillArgs fa{};
    if (!accumulate && grad->rows > 0 && grad->cols > 0) {
        const bool flat = grad->ld == grad->cols;
        fa = {static_cast<char*>(grad->data), flat ? 1 : (long long)grad->rows,
              (long long)grad->cols * es * (flat ? (long long)grad->rows : 1), (long long)grad->ld * es};
    }
    constexpr int smem = (SORT_WARPS * SORT_BINS + SORT_BINS + 32 + 4) * (int)sizeof(uint32_t);
    if (cudaFuncSetAttribute(k_sort_fill, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
        return ISO_ERR_CUDA;
    int fill_ctas = 0;
    if (fa.base) {
        const long long chunks = fa.rows * ((fa.width + FILL_CHUNK - 1) / FILL_CHUNK);
        fill_ctas = (int)std::min((chunks + SORT_WARPS - 1) / SORT_WARPS, (long long)train_sms());
        fill_ctas = (fill_ctas + SORT_CLUSTER - 1) / SORT_CLUSTER * SORT_CLUSTER;
    }
    TRAIN_LAUNCH((k_sort_fill<<<SORT_CLUSTER + fill_ctas, SORT_TPB, smem, s>>>(sa, fa)));
    if (n == 0 || grad->rows == 0 || grad->cols == 0) return ISO_OK;

    RowArgs ra;
    ra.sorted = sa.buf[0];
    ra.n = n;
    ra.rows = (uint32_t)grad->rows;
    ra.scale = scale;
    ra.cols = (int)grad->cols;
    ra.segs = (int)((grad->cols + TRAIN_SEG - 1) / TRAIN_SEG);
    ra.accumulate = accumulate;
    ra.part = reinterpret_cast<float*>(ws + L.part);
    ra.ld_part = L.ld_part;
    ra.joins = reinterpret_cast<uint32_t*>(ws + L.joins);
    ra.n_joins = sa.n_joins;
    const long long wins = (n + WIN - 1) / WIN;
    const int sums_grid = (int)std::min((wins * ra.segs + EM_WPB - 1) / EM_WPB, (long long)train_sms() * 8);
    const int join_grid = (int)std::min(wins * ((grad->cols + JOIN_COLS - 1) / JOIN_COLS), (long long)train_sms() * 2);
    return dispatch2(dY->dtype, grad->dtype, rows_aligned(dY) && rows_aligned(grad), [&](auto* tp, auto* op, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        constexpr bool VEC = decltype(v)::value;
        TRAIN_LAUNCH((k_row_sums<T, O, VEC><<<sums_grid, EM_TPB, 0, s>>>(
            static_cast<const T*>(dY->data), dY->ld, static_cast<O*>(grad->data), grad->ld, ra)));
        if (wins > 1)
            TRAIN_LAUNCH((k_row_join<O, VEC><<<join_grid, JOIN_TPB, 0, s>>>(static_cast<O*>(grad->data), grad->ld, ra)));
        return ISO_OK;
    });
}

}  // extern "C"
