// iso_embed.cu -- the token embedding and its gradient by sorted tokens.
//
// Forward: a gather of table rows, bound by HBM; a warp takes up to 1024
// channels of one token, all its loads in flight at once.
//
// Gradient: grad[v] = scale * sum of dY[t] over the tokens of id v.
//   k_sort       one cluster of eight CTAs (one CTA for fewer tokens) sorts
//                (id, token) by a stable LSD radix sort, digits of up to nine
//                bits; a short list is sorted by counting;
//   k_fill       writes the zeros of a gradient that is not accumulated.  A
//                vocabulary has far more rows than a batch has tokens, so this
//                is the bulk of the traffic; it runs beside the sort (started
//                early, or, when it is short, by other CTAs of the sort's grid)
//                and hides it.  Rows with tokens are written a second time;
//   k_row_sums   the sorted tokens in windows of equal length: a warp adds a
//                window's dY rows over 256 channels and writes the sum of
//                every run of equal ids that lies inside the window; a run
//                that crosses a window's edge leaves one partial row a window;
//   k_row_join   the runs that cross windows: partials added, row written.
// Up to 32 tokens, k_grad_few does it all in one launch: a lane holds a token's
// id, and a warp writes its rows once each, with the tokens a ballot finds.
// Sums are binary32 and their order is fixed by the sorted positions and the
// window length (a function of the sizes alone), so equal inputs give equal
// bits, and a frequent id's sum is a short tree, not one long chain.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace iso {
namespace {

constexpr int EM_TPB = 128;
constexpr int EM_WPB = EM_TPB / 32;
constexpr int EM_SEGS = 4;                              // segments of one token a warp takes

constexpr int SORT_CLUSTER = 8;
constexpr int SORT_TPB = 1024;
constexpr int SORT_WARPS = SORT_TPB / 32;
constexpr int SORT_BITS = 9;
constexpr int SORT_BINS = 1 << SORT_BITS;
// Up to this many tokens one CTA sorts alone.  Measured, the accumulating gradient
// of 152064 x 64 whole, one CTA against a cluster of eight: 2000 tokens 23.1 / 23.2
// us, 4096 tokens 29.5 / 24.1 us.
constexpr long long SORT_ONE_CTA = 2048;
constexpr int SORT_SMEM = (SORT_WARPS * SORT_BINS + SORT_BINS + 32 + 4) * (int)sizeof(uint32_t);
constexpr int FILL_TPB = 256;
constexpr int FILL_CHUNK = 8192;                        // bytes of zeros a warp writes
// Up to this many tokens are sorted by counting: the longest list at which that
// led for every table.  Measured, the accumulating gradient of 64 columns whole,
// that against the radix sort: 256 tokens of 500 rows (one pass) 11.5 / 12.5 us,
// of 152064 rows (two) 11.5 / 14.8; 333 tokens 12.8 / 12.7 and 12.9 / 15.3; 512
// tokens 15.3 / 13.5 and 15.2 / 16.4; 1000 tokens 30 / 16 and 29 / 19.  So where
// the radix sort takes two passes the limit could be near 512.
constexpr int SORT_RANK = 256;
// Up to this many chunks the zeros ride along with the sort of one CTA: one launch
// less (about 3 us of host time); 32 MB take about 5 us there.
constexpr long long FILL_WITH_SORT = (32 << 20) / FILL_CHUNK;
constexpr int SUM_TPB = 128;
constexpr int SUM_WPB = SUM_TPB / 32;
constexpr int SUM_RING = 4096;                          // bytes of dY rows in flight per warp
// Windows are as long as leaves this many warps: 24 for each of a GB300's 152
// SMs.  A constant, whatever GPU runs: the order of the sums is the windows'.
constexpr long long SUM_WARPS = 152 * 24;
constexpr int WIN_MIN = 8, WIN_MAX = 256;
// Up to this many tokens take k_grad_few.  Measured, it against the sort and
// the rest: 1 token, 18992 x 192 f32 4.5 / 8.3 us, 151936 x 1536 bf16 63 / 67 us;
// 32 tokens 5.5 / 12.0 and 63 / 71 us.
constexpr int GF_TOKENS = 32;
constexpr int GF_TPB = 128;
constexpr int GF_WARPS = GF_TPB / 32;
constexpr int GF_SEGS = 4;                              // segments of a row a warp takes
constexpr int GF_BYTES = 4096;                          // of gradient a warp writes, about
constexpr int JOIN_TPB = 128;
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
                                                  long long ldo, int cols, int runs, int32_t* status) {
    const int lane = threadIdx.x & 31;
    const long long items = ids.n * runs;
    for (long long i = (long long)blockIdx.x * EM_WPB + (threadIdx.x >> 5); i < items; i += (long long)gridDim.x * EM_WPB) {
        const long long t = i / runs;
        const int c0 = (int)(i - t * runs) * (EM_SEGS * TRAIN_SEG), c = c0 + lane * 8;
        const long long id = load_id(ids, t);
        const bool in = id != ids.pad_id && id >= 0 && id < ids.rows;
        if (!in && id != ids.pad_id && status && lane == 0) *status = ISO_ERR_INDEX;
        const int full = VEC ? min(EM_SEGS, (cols - c0) / TRAIN_SEG) : 0;
        const T* src = table + (in ? id : 0) * ldt;
        O* dst = out + t * ldo;
        Raw8<T> raw[EM_SEGS];
#pragma unroll
        for (int k = 0; k < EM_SEGS; ++k)
            if (VEC && k < full && in) raw[k].load(src + c + k * TRAIN_SEG);
#pragma unroll
        for (int k = 0; k < EM_SEGS; ++k) {
            float v[8] = {};
            if (VEC && k < full) {
                if (in) raw[k].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= scale;
                put8(dst + c + k * TRAIN_SEG, v);
            } else if (c0 + k * TRAIN_SEG < cols) {
                if (in) load8<VEC>(src, c + k * TRAIN_SEG, cols, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= scale;
                store8<VEC>(dst, c + k * TRAIN_SEG, cols, v);
            }
        }
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

// zeros in short blocks, in the order of addresses (a persistent grid reaches
// 6.4 - 6.6 TB/s of writes here, short blocks 7.7)
__device__ __forceinline__ void fill_zeros(const FillArgs& f, long long warp, long long warps, int lane) {
    const long long per_row = (f.width + FILL_CHUNK - 1) / FILL_CHUNK;
    for (long long i = warp; i < f.rows * per_row; i += warps) {
        const long long r = i / per_row, off = (i - r * per_row) * FILL_CHUNK;
        warp_zero(f.base + r * f.stride + off, min((long long)FILL_CHUNK, f.width - off), lane);
    }
}
__global__ void __launch_bounds__(FILL_TPB) k_fill(FillArgs f) {
    fill_zeros(f, (long long)blockIdx.x * (FILL_TPB / 32) + (threadIdx.x >> 5), (long long)gridDim.x * (FILL_TPB / 32),
               threadIdx.x & 31);
    // this grid is not done before the sort that it started beside
    if (blockIdx.x == gridDim.x - 1) wait_before();
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

// The list of a few tokens sorted by counting: a token's place is the number of
// tokens with a smaller id, or the same id and a smaller position.
__device__ __forceinline__ void rank_sort(const SortArgs& a, uint32_t* keys, int warp, int lane) {
    const int n = (int)a.ids.n, t = threadIdx.x, padded = (n + 31) / 32 * 32;
    bool bad = false;
    uint2 it = make_uint2(0xFFFFFFFFu, 0u);                  // past the list: after every id
    if (t < n) it = sort_item(a, nullptr, t, bad);
    if (t < padded) keys[t] = it.x;
    const int any = __syncthreads_or(bad);
    if (t == 0) {
        if (a.status) *a.status = any ? (int32_t)ISO_ERR_INDEX : (int32_t)ISO_OK;
        *a.n_joins = 0;
    }
    if (warp * 32 >= n) return;
    uint32_t rank = 0;
    for (int tile = 0; tile < padded / 32; ++tile) {
        const uint4* k4 = reinterpret_cast<const uint4*>(keys + tile * 32);
        if (tile == warp) {
#pragma unroll
            for (int j = 0; j < 32; ++j) rank += keys[tile * 32 + j] < it.x + (j < lane ? 1u : 0u);
        } else {
            const uint32_t below = it.x + (tile < warp ? 1u : 0u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 k = k4[j];
                rank += (k.x < below) + (k.y < below) + (k.z < below) + (k.w < below);
            }
        }
    }
    if (t < n) a.buf[0][rank] = it;
}

// CTAS: the CTAs of the one cluster that sorts.  With CTAS = 1 further CTAs of
// the grid may write the zeros f.
template <int CTAS>
__global__ void __launch_bounds__(SORT_TPB, 1) k_sort(SortArgs a, FillArgs f) {
    start_next();                                                     // the fill, or the row sums, may start
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (CTAS == 1 && blockIdx.x > 0) {
        fill_zeros(f, (long long)(blockIdx.x - 1) * SORT_WARPS + warp, (long long)(gridDim.x - 1) * SORT_WARPS, lane);
        return;
    }
    extern __shared__ __align__(16) uint32_t sort_smem[];
    if (CTAS == 1 && a.ids.n <= SORT_RANK) {
        rank_sort(a, sort_smem, warp, lane);
        return;
    }
    uint32_t* const cnt = sort_smem;                                  // [warp][bin]
    uint32_t* const tot = cnt + SORT_WARPS * SORT_BINS;               // [bin]: this CTA's items
    uint32_t* const scan = tot + SORT_BINS;                           // [warp sums]
    int* const bad_flag = reinterpret_cast<int*>(scan + 32);
    cg::cluster_group cluster = cg::this_cluster();
    auto sync_all = [&] { if (CTAS == 1) __syncthreads(); else cluster.sync(); };
    const int me = CTAS == 1 ? 0 : (int)cluster.block_rank();
    const uint32_t lt = (1u << lane) - 1u;
    // every warp owns a contiguous range of positions, in order, so that ranks
    // counted range by range are stable
    const long long n = a.ids.n;
    const long long per = ((n + CTAS * SORT_WARPS - 1) / (CTAS * SORT_WARPS) + 31) / 32 * 32;
    const long long t0 = min(n, ((long long)me * SORT_WARPS + warp) * per), t1 = min(n, t0 + per);
    // warps of this CTA that have items
    const long long cta0 = min(n, (long long)me * SORT_WARPS * per);
    const int warps = per ? (int)min((long long)SORT_WARPS, (n - cta0 + per - 1) / per) : 0;
    const int bins = 1 << a.bits;
    if (threadIdx.x == 0) *bad_flag = 0;
    __syncthreads();
    bool bad = false;
    for (int p = 0; p < a.passes; ++p) {
        const uint2* src = p == 0 ? nullptr : a.buf[(a.passes - p) & 1];
        uint2* dst = a.buf[(a.passes - 1 - p) & 1];
        const int shift = p * a.bits;
        const uint32_t mask = (uint32_t)bins - 1u;
        uint32_t* const mine = cnt + warp * SORT_BINS;
        if (warp < warps)
            for (int i = lane; i < bins; i += 32) mine[i] = 0;
        __syncwarp();
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
        if (threadIdx.x < bins) {
            uint32_t s = 0;
#pragma unroll 8
            for (int w = 0; w < warps; ++w) {
                const uint32_t v = cnt[w * SORT_BINS + threadIdx.x];
                cnt[w * SORT_BINS + threadIdx.x] = s;
                s += v;
            }
            tot[threadIdx.x] = s;
        }
        sync_all();
        // start of each bin for this CTA: earlier bins of all CTAs, earlier CTAs of this bin
        uint32_t all = 0, before = 0;
        if (threadIdx.x < bins) {
#pragma unroll
            for (int c = 0; c < CTAS; ++c) {
                const uint32_t v = CTAS == 1 ? tot[threadIdx.x] : cluster.map_shared_rank(tot, c)[threadIdx.x];
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
        if (threadIdx.x < bins) {
            uint32_t base = before + inc - all;
            for (int w = 0; w < warp; ++w) base += scan[w];
#pragma unroll 8
            for (int w = 0; w < warps; ++w) cnt[w * SORT_BINS + threadIdx.x] += base;
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
            for (int c = 0; c < CTAS; ++c) any |= CTAS == 1 ? *bad_flag : *cluster.map_shared_rank(bad_flag, c);
            if (a.status) *a.status = any ? (int32_t)ISO_ERR_INDEX : (int32_t)ISO_OK;
            *a.n_joins = 0;
        }
        sync_all();   // dst is complete; no CTA still reads another's shared memory
    }
}

struct RowArgs {
    const uint2* sorted;
    long long n;
    uint32_t rows;          // table rows: the id of padding
    float scale;
    int cols, segs, accumulate;
    int win;                // sorted tokens per window
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
    if (VEC && c + 8 <= cols) put8(row + c, v);
    else store8<false>(row, c, cols, v);
}

// eight channels of a row of dY into this lane's place in shared memory,
// channels past the end as zeros
template <typename T>
__device__ __forceinline__ void copy8_async(uint32_t dst, const T* row, int c, int cols) {
    const int bytes = max(0, min(8, cols - c)) * (int)sizeof(T);
    const char* src = reinterpret_cast<const char*>(row + (bytes ? c : 0));
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const int here = max(0, min(16, bytes - 16 * i));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                     :: "r"(dst + 16u * i), "l"(src + (here ? 16 * i : 0)), "r"(here) : "memory");
    }
}

// A warp per (window, 256 channels).  Rows of dY that start on 16-byte
// boundaries stream through a ring of rows in shared memory (every
// lane reads back what it copied itself), so the loads of later tokens are
// under way while a run is written; loaded eight tokens at a time into
// registers instead, the 32768 x 3584 case measured 148 us, this way 75 us (84
// us with blocks of 256 threads).
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(SUM_TPB) k_row_sums(const T* dy, long long ldd, O* grad, long long ldg, RowArgs a) {
    start_next();
    wait_before();
    constexpr int LANE_BYTES = 8 * (int)sizeof(T), SLOT = 32 * LANE_BYTES, DEPTH = SUM_RING / SLOT;
    __shared__ __align__(16) unsigned char ring[VEC ? SUM_WPB * SUM_RING : 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned char* const mine = ring + (VEC ? warp * SUM_RING + lane * LANE_BYTES : 0);
    const uint32_t mine_s = smem_u32(mine);
    const long long wins = (a.n + a.win - 1) / a.win, items = wins * a.segs;
    for (long long i = (long long)blockIdx.x * SUM_WPB + warp; i < items; i += (long long)gridDim.x * SUM_WPB) {
        const long long w = i / a.segs;
        const int seg = (int)(i - w * a.segs), c = seg * TRAIN_SEG + lane * 8;
        const long long p0 = w * a.win, end = min(a.n, p0 + a.win);
        // lane l holds sorted item 32 q + l of the window, for this q and the next
        auto items_at = [&](long long p) { return p + lane < end ? a.sorted[p + lane] : make_uint2(a.rows, 0u); };
        uint2 cur = items_at(p0), nxt = items_at(p0 + 32);
        const uint32_t prev = p0 > 0 ? a.sorted[p0 - 1].x : 0xFFFFFFFFu;
        const uint32_t after = end < a.n ? a.sorted[end].x : 0xFFFFFFFFu;
        auto id_at = [&](int k) { return __shfl_sync(0xFFFFFFFFu, k < 32 ? cur.x : nxt.x, k & 31); };
        auto pos_at = [&](int k) { return __shfl_sync(0xFFFFFFFFu, k < 32 ? cur.y : nxt.y, k & 31); };
        auto fetch = [&](int k, uint32_t slot) {                     // start the copy of item k (padding: nothing)
            if (VEC) {
                const uint32_t id = id_at(k), pos = pos_at(k);
                if (id < a.rows) copy8_async(mine_s + slot * SLOT, dy + (long long)pos * ldd, c, a.cols);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        };
        float acc[8] = {};
        uint32_t id = id_at(0);
        bool enters = id == prev;
#pragma unroll 1
        for (int k = 0; k < DEPTH - 1; ++k) fetch(k, (uint32_t)k);
        uint32_t slot = 0;
        for (long long q = p0; id < a.rows; q += 32) {               // padding sorts last
#pragma unroll 1
            for (int k = 0; k < 32 && id < a.rows; ++k) {
                const uint32_t next = id_at(k + 1);
                fetch(k + DEPTH - 1, (slot + DEPTH - 1) % DEPTH);
                float v[8];
                if constexpr (VEC) {
                    asm volatile("cp.async.wait_group %0;" :: "n"(DEPTH - 1) : "memory");
                    Raw8<T> raw;
                    raw.load_shared(mine + slot * SLOT);
                    raw.get(v);
                } else {
                    load8<false>(dy + (long long)pos_at(k) * ldd, c, a.cols, v);
                }
                slot = (slot + 1) % DEPTH;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += v[j];
                // past the window's end, ids read as padding
                const bool leaves = q + k + 1 == end && after == id;
                if (next != id) {
                    if (!enters && !leaves)
                        write_row<O, VEC>(grad + (long long)id * ldg, c, a.cols, acc, a.scale, a.accumulate);
                    else if (c < a.cols)
                        put8(a.part + (w * 2 + (enters ? 0 : 1)) * a.ld_part + c, acc);
                    if (!enters && leaves && seg == 0 && lane == 0) a.joins[atomicAdd(a.n_joins, 1u)] = (uint32_t)w;
                    enters = false;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
                }
                id = next;
            }
            cur = nxt;
            nxt = items_at(q + 64);
        }
        if (VEC) asm volatile("cp.async.wait_all;" ::: "memory");
    }
}

// A CTA per (run, 128 channels): its warps take the run's partial rows in turn.
template <typename O>
__global__ void __launch_bounds__(JOIN_TPB) k_row_join(O* grad, long long ldg, RowArgs a) {
    __shared__ float4 sums[JOIN_TPB / 32][32];
    wait_before();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int WARPS = JOIN_TPB / 32;
    const int slices = (a.cols + JOIN_COLS - 1) / JOIN_COLS;
    const long long items = (long long)*a.n_joins * slices, wins = (a.n + a.win - 1) / a.win;
    for (long long i = blockIdx.x; i < items; i += gridDim.x) {
        const long long e = i / slices, w = a.joins[e];
        const int c = (int)(i - e * slices) * JOIN_COLS + lane * 4;
        const uint32_t id = a.sorted[(w + 1) * a.win].x;
        // windows w + 1 .. w + k whose first token continues the run
        long long k = 0;
        for (;;) {
            const long long q = w + 1 + k + threadIdx.x;
            const int got = __syncthreads_count(q < wins && a.sorted[q * a.win].x == id);
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

// The gradient for few tokens: a warp takes `rows_per` rows, up to 1024 channels
// of them, and adds a row's tokens in ascending order.  Accumulating, it takes
// the row of one token instead, if no earlier token has it.
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(GF_TPB) k_grad_few(const T* dy, long long ldd, O* grad, long long ldg, Ids ids,
                                                     float scale, int cols, int runs, int rows_per, int accumulate,
                                                     int32_t* status) {
    const int lane = threadIdx.x & 31;
    const long long id = lane < ids.n ? load_id(ids, lane) : ids.pad_id;
    const bool in = lane < ids.n && id != ids.pad_id && id >= 0 && id < ids.rows;
    if (status && blockIdx.x == 0 && threadIdx.x < 32) {
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, !in && id != ids.pad_id);
        if (lane == 0) *status = bad ? (int32_t)ISO_ERR_INDEX : (int32_t)ISO_OK;
    }
    const long long items = (accumulate ? ids.n : (ids.rows + rows_per - 1) / rows_per) * runs;
    for (long long i = (long long)blockIdx.x * GF_WARPS + (threadIdx.x >> 5); i < items; i += (long long)gridDim.x * GF_WARPS) {
        const long long q = i / runs, first = __shfl_sync(0xFFFFFFFFu, id, (int)(q & 31));
        const int c0 = (int)(i - q * runs) * (GF_SEGS * TRAIN_SEG);
        const long long row0 = accumulate ? first : q * rows_per;
        const int rows = accumulate ? 1 : (int)min((long long)rows_per, ids.rows - row0);
        const uint32_t here = __ballot_sync(0xFFFFFFFFu, in && id >= row0 && id < row0 + rows);
        if (accumulate && (here == 0 || __ffs(here) - 1 != (int)q)) continue;
        for (int r = 0; r < rows; ++r) {
            const uint32_t tokens = here ? __ballot_sync(0xFFFFFFFFu, in && id == row0 + r) : 0u;
            O* row = grad + (row0 + r) * ldg;
            for (int c = c0 + lane * 8; c - lane * 8 < min(cols, c0 + GF_SEGS * TRAIN_SEG); c += TRAIN_SEG) {
                float acc[8] = {};
                if (tokens) {
                    for (uint32_t m = tokens; m; m &= m - 1) {
                        float v[8];
                        load8<VEC>(dy + (long long)(__ffs(m) - 1) * ldd, c, cols, v);
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[j] += v[j];
                    }
                    write_row<O, VEC>(row, c, cols, acc, scale, accumulate);
                } else if (VEC && c + 8 <= cols) {
                    put8(row + c, acc);
                } else {
                    store8<false>(row, c, cols, acc);
                }
            }
        }
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

// Sorted tokens per window: short enough for SUM_WARPS warps (one wave of
// k_row_sums), within WIN_MIN .. WIN_MAX.
int window_of(int64_t n, int64_t cols) {
    const long long segs = (cols + TRAIN_SEG - 1) / TRAIN_SEG;
    int win = WIN_MIN;
    while (win < WIN_MAX && n * segs > SUM_WARPS * win) win *= 2;
    return win;
}

// workspace: header (join count), the two sort buffers, the join list, the partial rows
struct GradLayout {
    size_t buf0, buf1, joins, part, end;
    long long ld_part;
    int win;
};
GradLayout grad_layout(int64_t n, int64_t cols) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    GradLayout L{};
    if (n <= GF_TOKENS) {            // k_grad_few needs none
        L.end = 256;
        return L;
    }
    L.win = window_of(n, cols);
    const size_t wins = (size_t)((n + L.win - 1) / L.win);
    L.ld_part = (cols + 7) / 8 * 8;
    L.buf0 = 256;
    L.buf1 = L.buf0 + up((size_t)n * sizeof(uint2));
    L.joins = L.buf1 + up((size_t)n * sizeof(uint2));
    L.part = L.joins + up(wins * sizeof(uint32_t));
    L.end = L.part + up(wins * 2 * (size_t)L.ld_part * sizeof(float));
    return L;
}

long long fill_chunks(const FillArgs& f) { return f.base ? f.rows * ((f.width + FILL_CHUNK - 1) / FILL_CHUNK) : 0; }

// the sort: one cluster, and with CTAS = 1 the CTAs that write f's zeros
template <int CTAS>
int launch_sort(const SortArgs& a, const FillArgs& f, cudaStream_t s) {
    static std::atomic<uint64_t> ready{0};      // devices whose limit is raised, one bit each
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return ISO_ERR_CUDA;
    if (dev >= 64 || !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaFuncSetAttribute(k_sort<CTAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, SORT_SMEM) != cudaSuccess)
            return ISO_ERR_CUDA;
        if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CTAS + std::min((fill_chunks(f) + SORT_WARPS - 1) / SORT_WARPS, (long long)train_sms())));
    cfg.blockDim = dim3(SORT_TPB);
    cfg.dynamicSmemBytes = SORT_SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = CTAS;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    TRAIN_LAUNCH(cudaLaunchKernelEx(&cfg, k_sort<CTAS>, a, f));
    return ISO_OK;
}
// the zeros, allowed to start once the sort has
int launch_fill(const FillArgs& f, cudaStream_t s) {
    const long long chunks = fill_chunks(f);
    TRAIN_LAUNCH(launch_early(k_fill, (unsigned)std::min((chunks + FILL_TPB / 32 - 1) / (FILL_TPB / 32), (long long)EXTENT_LIMIT),
                              FILL_TPB, 0, s, f));
    return ISO_OK;
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
    const int runs = (int)((out->cols + EM_SEGS * TRAIN_SEG - 1) / (EM_SEGS * TRAIN_SEG));
    const unsigned grid = (unsigned)std::min(((long long)n * runs + EM_WPB - 1) / EM_WPB, (long long)EXTENT_LIMIT);
    return dispatch2(table->dtype, out->dtype, rows_aligned(table) && rows_aligned(out), [&](auto* tp, auto* op, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        TRAIN_LAUNCH((k_embed<T, O, decltype(v)::value><<<grid, EM_TPB, 0, s>>>(
            static_cast<const T*>(table->data), table->ld, id, scale, static_cast<O*>(out->data), out->ld,
            (int)out->cols, runs, status)));
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
    const Ids list{ids, (long long)n, (long long)pad_id, (long long)grad->rows, ids_i64};
    const int es = elem_size(grad->dtype);
    const bool vec = rows_aligned(dY) && rows_aligned(grad);
    if (grad->rows == 0 || grad->cols == 0)
        return !status || cudaMemsetAsync(status, 0, sizeof(int32_t), s) == cudaSuccess ? ISO_OK : ISO_ERR_CUDA;
    if (n <= GF_TOKENS) {
        const long long width = std::min((long long)grad->cols, (long long)GF_SEGS * TRAIN_SEG) * es;
        const int rows_per = (int)std::max(1LL, GF_BYTES / width);
        const int runs = (int)((grad->cols + GF_SEGS * TRAIN_SEG - 1) / (GF_SEGS * TRAIN_SEG));
        const long long items = (accumulate ? std::max<long long>(n, 1) : (grad->rows + rows_per - 1) / rows_per) * runs;
        const unsigned grid = (unsigned)std::min((items + GF_WARPS - 1) / GF_WARPS, (long long)EXTENT_LIMIT);
        return dispatch2(dY->dtype, grad->dtype, vec, [&](auto* tp, auto* op, auto v) -> int {
            using T = std::remove_pointer_t<decltype(tp)>;
            using O = std::remove_pointer_t<decltype(op)>;
            TRAIN_LAUNCH((k_grad_few<T, O, decltype(v)::value><<<grid, GF_TPB, 0, s>>>(
                static_cast<const T*>(dY->data), dY->ld, static_cast<O*>(grad->data), grad->ld, list, scale,
                (int)grad->cols, runs, rows_per, accumulate, status)));
            return ISO_OK;
        });
    }

    SortArgs sa;
    sa.ids = list;
    sa.buf[0] = reinterpret_cast<uint2*>(ws + L.buf0);
    sa.buf[1] = reinterpret_cast<uint2*>(ws + L.buf1);
    int bits = 1;                                            // ids 0 .. rows, rows marking padding
    while (bits < 31 && ((int64_t)grad->rows >> bits)) ++bits;
    sa.passes = (bits + SORT_BITS - 1) / SORT_BITS;
    sa.bits = (bits + sa.passes - 1) / sa.passes;
    sa.status = status;
    sa.n_joins = reinterpret_cast<uint32_t*>(ws);
    FillArgs fa{};
    if (!accumulate) {
        const bool flat = grad->ld == grad->cols;
        fa = {static_cast<char*>(grad->data), flat ? 1 : (long long)grad->rows,
              (long long)grad->cols * es * (flat ? (long long)grad->rows : 1), (long long)grad->ld * es};
    }
    if (n <= SORT_ONE_CTA && fill_chunks(fa) <= FILL_WITH_SORT) {
        ISO_TRY(launch_sort<1>(sa, fa, s));
    } else {
        ISO_TRY(n <= SORT_ONE_CTA ? launch_sort<1>(sa, FillArgs{}, s) : launch_sort<SORT_CLUSTER>(sa, FillArgs{}, s));
        if (fa.base) ISO_TRY(launch_fill(fa, s));
    }

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
    ra.win = L.win;
    const long long wins = (n + L.win - 1) / L.win;
    const int sums_grid = (int)std::min((wins * ra.segs + SUM_WPB - 1) / SUM_WPB, (long long)EXTENT_LIMIT);
    const int join_grid = (int)std::min(wins * ((grad->cols + JOIN_COLS - 1) / JOIN_COLS), (long long)train_sms() * 16);
    return dispatch2(dY->dtype, grad->dtype, vec, [&](auto* tp, auto* op, auto v) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        constexpr bool VEC = decltype(v)::value;
        TRAIN_LAUNCH(launch_early(k_row_sums<T, O, VEC>, (unsigned)sums_grid, SUM_TPB, 0, s, static_cast<const T*>(dY->data),
                                  dY->ld, static_cast<O*>(grad->data), grad->ld, ra));
        if (wins > 1)
            TRAIN_LAUNCH(launch_early(k_row_join<O>, (unsigned)join_grid, JOIN_TPB, 0, s, static_cast<O*>(grad->data),
                                      grad->ld, ra));
        return ISO_OK;
    });
}

}  // extern "C"
