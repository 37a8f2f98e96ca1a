// iso_wgrad.cu -- the weight gradient G = dY^T X_hat from a checkpoint, on the
// fifth-generation tensor cores.
//
// Both operands are row-major with tokens in rows, so the contraction runs
// over rows: their tiles are "MN-major" (64 channels of one token contiguous),
// which tcgen05.mma takes from shared memory as it takes K-major ones, and no
// transposition is needed.
//   operands   X_hat is decoded to bf16 (exact: codes are integers below 2^8,
//              scales powers of two) into the workspace.  A bf16 dY is read in
//              place when its rows start on 16-byte boundaries, else copied.
//              A binary32 dY is split into three bf16 parts of eight
//              significant bits each, hi + mid + lo = dY, and G is the sum of
//              the three products; so every product is exact and sums are
//              binary32.
//   k_wgrad    a pair of CTAs per 256 x 256 tile of G, 64 tokens per stage
//              (16 KB of each operand per CTA, six stages), accumulated in
//              tensor memory, two accumulators so that one tile's epilogue
//              overlaps the next tile's products; persistent over the tiles.
//   split      a G of few tiles under many tokens is cut along the tokens as
//              well; the parts are binary32 in the workspace and k_wgrad_join
//              adds them in order.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>

namespace iso {
namespace {

constexpr int WG_BM = 256;                 // rows of G (dY channels) per CTA pair
constexpr int WG_BN = 256;                 // columns of G (X channels) per CTA pair
constexpr int WG_BK = 64;                  // tokens per stage
constexpr int WG_STAGES = 6;
constexpr int WG_BOX = 64;                 // channels of one copy: 128 bytes, the swizzle's row
constexpr int WG_BOX_BYTES = WG_BOX * WG_BK * 2;
constexpr int WG_OP_BYTES = 2 * WG_BOX_BYTES;          // 128 channels of an operand: this CTA's half
constexpr int WG_STAGE_BYTES = 2 * WG_OP_BYTES;
constexpr int WG_SMEM = 1024 + WG_STAGES * WG_STAGE_BYTES + 256;
constexpr int WG_EPI_WARPS = 8;
constexpr int WG_THREADS = (WG_EPI_WARPS + 2) * 32;    // epilogue warps, a copy warp, a product warp
constexpr int WG_MAX_PARTS = 3;
constexpr int WG_MAX_SPLIT = 8;
constexpr int WG_BAND = 8;                 // tile rows that are walked together

struct WgradArgs {
    int32_t M, N;
    int32_t m_tiles, n_tiles;
    int32_t k_tiles;       // steps of the whole contraction: parts x ceil(tokens / 64)
    int32_t parts;
    int32_t split;
    int32_t accumulate;
    void* out;             // split = 1: G
    long long ldo;
    int32_t out_dtype;
    int32_t out_vec;       // rows of G start on 16-byte boundaries
    float* part;           // split > 1: [split][M][ld_part]
    long long ld_part;
    int32_t* status;
};
struct WgradMaps {
    CUtensorMap a[WG_MAX_PARTS], b;
};

// Shared-memory descriptor of an MN-major operand in the 128-byte swizzle:
// 64 channels (128 bytes) by eight tokens make an atom of 1024 bytes; the next
// eight tokens follow it, the next 64 channels are one copy box further on.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)((WG_BOX_BYTES >> 4) & 0x3FFF) << 16;    // leading offset: 64 channels on
    d |= (uint64_t)((1024u >> 4) & 0x3FFFu) << 32;          // stride offset: eight tokens on
    d |= (uint64_t)1u << 46;
    d |= (uint64_t)2u << 61;
    return d;
}

// kind::f16, fp32 accumulator, bf16 A and B, both MN-major, M = 256 over the
// pair, N = 256
constexpr uint32_t WG_IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) |
                              ((uint32_t)(WG_BN >> 3) << 17) | ((uint32_t)(WG_BM >> 4) << 24);

__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// the address of CTA 0's copy of a shared-memory object of this CTA
__device__ __forceinline__ uint32_t in_leader(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a tile into this CTA's shared memory, its bytes counted on a barrier of the pair
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_bf16_pair(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(tmem_d), "l"(a), "l"(b), "r"(WG_IDESC), "r"(accumulate) : "memory");
}
// arrive on this barrier in both CTAs once the products issued so far are done
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "n"(MBAR_PROBE_NS) : "memory");
    return ok != 0;
}
// bounded wait; false once the limit is reached or another thread of the CTA gave up
__device__ __forceinline__ bool wait_pair(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    for (int spin = 0; spin < MBAR_SPIN_LIMIT; ++spin) {
        if (try_wait_cluster(bar, parity)) return true;
        if ((spin & 1023) == 1023 && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}
__device__ __forceinline__ void tmem_load32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                   "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
                   "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of one row of G from column n
template <typename O>
__device__ __forceinline__ void store_row32(O* row, int n, int N, float (&v)[32], bool vec, int accumulate) {
    if (vec && n + 32 <= N) {
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = v[j + k];
            if (accumulate) {
                float old[8];
                load8<true>(row, n + j, N, old);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] += old[k];
            }
            store8<true>(row, n + j, N, w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (n + j < N) from_f32(accumulate ? to_f32(row[n + j]) + v[j] : v[j], row[n + j]);
    }
}

// Work item i: a part of the contraction of one tile; tiles in bands of
// WG_BAND tile rows, column by column inside a band, so that the pairs that
// run together share their operands' rows in L2.
__device__ __forceinline__ void work_item(const WgradArgs& g, int i, int& m0, int& n0, int& k0, int& k1, int& part) {
    const int tile = i / g.split;
    part = i - tile * g.split;
    const int band = tile / (WG_BAND * g.n_tiles), in = tile - band * WG_BAND * g.n_tiles;
    const int rows = min(WG_BAND, g.m_tiles - band * WG_BAND);
    m0 = (band * WG_BAND + in % rows) * WG_BM;
    n0 = in / rows * WG_BN;
    k0 = (int)((long long)g.k_tiles * part / g.split);
    k1 = (int)((long long)g.k_tiles * (part + 1) / g.split);
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WG_THREADS, 1)
k_wgrad(const __grid_constant__ WgradMaps maps, WgradArgs g) {
    extern __shared__ unsigned char wg_smem_raw[];
    unsigned char* const smem =
        reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(wg_smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + WG_STAGES * WG_STAGE_BYTES);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * WG_STAGES + 4);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const uint32_t st = smem_u32(smem), bar = smem_u32(bars);
    auto full = [&](int s) { return bar + 8u * s; };                          // leader: both CTAs' copies landed
    auto empty = [&](int s) { return bar + 8u * (WG_STAGES + s); };           // products that read the stage are done
    auto acc_full = [&](int a) { return bar + 8u * (2 * WG_STAGES + a); };    // accumulator complete
    auto acc_empty = [&](int a) { return bar + 8u * (2 * WG_STAGES + 2 + a); };   // leader: accumulator read by all

    if (threadIdx.x == 0) {
        for (int s = 0; s < WG_STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(acc_full(a), 1);
            mbar_init(acc_empty(a), 2 * WG_EPI_WARPS);
        }
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_barrier();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int items = g.m_tiles * g.n_tiles * g.split;

    if (warp == WG_EPI_WARPS && lane == 0) {
        // copies: this CTA's 128 channels of either operand
        int it = 0;
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            m0 += (int)rank * 128;
            n0 += (int)rank * 128;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % WG_STAGES;
                if (!wait_pair(empty(s), ((uint32_t)(it / WG_STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                if (rank == 0) mbar_arrive_tx(full(s), 2 * WG_STAGE_BYTES);
                const int kt = k / g.parts, p = k - kt * g.parts, t = kt * WG_BK;
                const uint32_t fb = in_leader(full(s)), a = st + s * WG_STAGE_BYTES, b = a + WG_OP_BYTES;
                tma_load_pair(a, &maps.a[p], m0, t, fb);
                tma_load_pair(a + WG_BOX_BYTES, &maps.a[p], m0 + WG_BOX, t, fb);
                tma_load_pair(b, &maps.b, n0, t, fb);
                tma_load_pair(b + WG_BOX_BYTES, &maps.b, n0 + WG_BOX, t, fb);
            }
        }
        // every copy into this CTA has been consumed before it may exit: the
        // products that read a stage free it in both CTAs
        for (int q = max(0, it - WG_STAGES); q < it; ++q)
            for (int spin = 0; spin < MBAR_SPIN_LIMIT; ++spin)
                if (try_wait_cluster(empty(q % WG_STAGES), (uint32_t)(q / WG_STAGES) & 1u) || *abort_flag) break;
    } else if (warp == WG_EPI_WARPS + 1 && lane == 0 && rank == 0) {
        // products of the pair
        int it = 0, n_acc = 0;
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs, ++n_acc) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            const int acc = n_acc & 1;
            if (!wait_pair(acc_empty(acc), ((uint32_t)(n_acc >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            tc_after();
            const uint32_t d = tmem + acc * WG_BN;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % WG_STAGES;
                if (!wait_pair(full(s), (uint32_t)(it / WG_STAGES) & 1u, abort_flag)) { ok = false; break; }
                tc_after();
                const uint32_t a = st + s * WG_STAGE_BYTES, b = a + WG_OP_BYTES;
#pragma unroll
                for (int q = 0; q < WG_BK / 16; ++q)   // 16 tokens per product: two atoms of eight
                    umma_bf16_pair(d, mn_desc(a + 2048u * q), mn_desc(b + 2048u * q), (k > k0 || q > 0) ? 1u : 0u);
                umma_commit_pair(empty(s));
            }
            umma_commit_pair(acc_full(acc));
        }
    } else if (warp < WG_EPI_WARPS) {
        // epilogue: warp w reads tensor-memory lanes 32 (w mod 4) ..., 128 of the 256 columns
        const int quad = warp & 3, half = warp >> 2;
        int n_acc = 0;
        for (int i = pair; i < items; i += pairs, ++n_acc) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            const int acc = n_acc & 1;
            if (!wait_pair(acc_full(acc), (uint32_t)(n_acc >> 1) & 1u, abort_flag)) break;
            __syncwarp();
            tc_after();
            const int row = m0 + (int)rank * 128 + quad * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const int n = n0 + half * 128 + c * 32;
                float v[32];
                tmem_load32(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * WG_BN + half * 128 + c * 32), v);
                if (row < g.M && n < g.N) {
                    if (g.part)
                        store_row32(g.part + ((long long)part * g.M + row) * g.ld_part, n, g.N, v, true, 0);
                    else if (g.out_dtype == ISO_BF16)
                        store_row32(static_cast<__nv_bfloat16*>(g.out) + row * g.ldo, n, g.N, v, g.out_vec, g.accumulate);
                    else
                        store_row32(static_cast<float*>(g.out) + row * g.ldo, n, g.N, v, g.out_vec, g.accumulate);
                }
            }
            tc_before();
            __syncwarp();
            if (lane == 0) arrive_cluster(in_leader(acc_empty(acc)));
        }
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    cluster_barrier();       // neither CTA exits while the other's products or arrivals may touch it
    if (threadIdx.x == 0 && *abort_flag && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512) : "memory");
    }
}

// out (+)= the sum of the parts in order
template <typename O, bool VEC>
__global__ void __launch_bounds__(256) k_wgrad_join(const float* part, long long ld_part, int split, int M, int N,
                                                    O* out, long long ldo, int accumulate) {
    const int segs = (N + 7) / 8;
    const long long n = (long long)M * segs;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const long long row = i / segs;
        const int c = (int)(i - row * segs) * 8;
        float s[8] = {};
        for (int p = 0; p < split; ++p) {
            float v[8];
            load8<true>(part + ((long long)p * M + row) * ld_part, c, (int)ld_part, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += v[j];
        }
        O* o = out + row * ldo;
        if (accumulate) {
            float old[8];
            load8<VEC>(o, c, N, old);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += old[j];
        }
        store8<VEC>(o, c, N, s);
    }
}

// dY as bf16 parts with rows on 16-byte boundaries.  Parts of a binary32
// value are its leading eight significant bits, cut off (not rounded, so that
// none overflows), then those of the remainder, twice: 24 bits in all.  A NaN
// or an infinity stays in the first part.
template <typename T>
__global__ void __launch_bounds__(256) k_wgrad_parts(const T* dy, long long ldd, int tokens, int M,
                                                     __nv_bfloat16* out, long long ldo, long long part_stride) {
    const int segs = (M + 7) / 8;
    const long long n = (long long)tokens * segs;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const long long t = i / segs;
        const int c = (int)(i - t * segs) * 8;
        float v[8];
        load8<false>(dy + t * ldd, c, M, v);
        __nv_bfloat16* o = out + t * ldo;
        if constexpr (sizeof(T) == 2) {
            store8<true>(o, c, (int)ldo, v);
        } else {
#pragma unroll
            for (int p = 0; p < WG_MAX_PARTS; ++p) {
                float hi[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t b = __float_as_uint(v[j]);
                    if ((b & 0x7FFFFFFFu) > 0x7F800000u) b |= 0x400000u;     // a NaN stays one without its low bits
                    hi[j] = __uint_as_float(b & 0xFFFF0000u);
                    v[j] = (b & 0x7F800000u) == 0x7F800000u ? 0.0f : v[j] - hi[j];
                }
                store8<true>(o + p * part_stride, c, (int)ldo, hi);
            }
        }
    }
}

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
// rows x cols bf16, `ld` elements from row to row; channels and tokens past
// the end read as zero
int bf16_map(CUtensorMap* map, const void* base, long long rows, long long cols, long long ld) {
    EncodeTiled fn = encode_tiled();
    if (!fn) return ISO_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)WG_BOX, (cuuint32_t)WG_BK};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? ISO_OK
               : ISO_ERR_CUDA;
}

int check_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out) {
    ISO_TRY(check_mat(dY));
    ISO_TRY(check_act(pack));
    ISO_TRY(check_mat(out));
    if (dY->rows != pack->rows || out->rows != dY->cols || out->cols != pack->cols) return ISO_ERR_SHAPE;
    return ISO_OK;
}

// the pairs of CTAs that run at once on the current device
int resident_pairs() {
    static int pairs[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (!pairs[dev]) {
        if (cudaFuncSetAttribute(k_wgrad, cudaFuncAttributeMaxDynamicSharedMemorySize, WG_SMEM) != cudaSuccess) return 0;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(train_sms() / 2 * 2));
        cfg.blockDim = dim3(WG_THREADS);
        cfg.dynamicSmemBytes = WG_SMEM;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 2;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, k_wgrad, &cfg) != cudaSuccess || n <= 0) return 0;
        pairs[dev] = n;
    }
    return pairs[dev];
}

struct WgradPlan {
    size_t x_bf16, dy_parts, parts, end;
    long long ldx, ldd, ld_part;
    int m_tiles, n_tiles, k_tiles, split, n_parts;
    bool dy_direct;
};
// Host only, the same for the sizing call and the launch (the pair count of a
// GB300 stands in where there is no device).
WgradPlan plan_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    WgradPlan p;
    const long long T = dY->rows, M = out->rows, N = out->cols;
    p.n_parts = dY->dtype == ISO_F32 ? 3 : 1;
    p.dy_direct = dY->dtype == ISO_BF16 && (reinterpret_cast<uintptr_t>(dY->data) & 15u) == 0 && dY->ld % 8 == 0;
    p.m_tiles = (int)((M + WG_BM - 1) / WG_BM);
    p.n_tiles = (int)((N + WG_BN - 1) / WG_BN);
    p.k_tiles = (int)((T + WG_BK - 1) / WG_BK) * p.n_parts;
    const long long tiles = (long long)p.m_tiles * p.n_tiles, pairs = std::max(1, train_sms() / 2);
    // cut the tokens where the tiles leave half the pairs idle, eight steps a part at least
    p.split = (int)std::max(1LL, std::min({pairs / std::max(1LL, tiles), (long long)p.k_tiles / 8, (long long)WG_MAX_SPLIT}));
    p.ldx = (N + 7) / 8 * 8;
    p.ldd = (M + 7) / 8 * 8;
    p.ld_part = (N + 7) / 8 * 8;
    p.x_bf16 = 0;
    p.dy_parts = up((size_t)T * p.ldx * 2);
    p.parts = p.dy_parts + (p.dy_direct ? 0 : up((size_t)T * p.ldd * 2 * p.n_parts));
    p.end = p.parts + (p.split > 1 ? up((size_t)p.split * M * p.ld_part * 4) : 0) + 256;
    return p;
}

template <typename F>
int by_dtype(int32_t dtype, F&& f) {
    return dtype == ISO_BF16 ? f((__nv_bfloat16*)nullptr) : f((float*)nullptr);
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_act_wgrad_workspace_size(const iso_mat* dY, const iso_act* pack, const iso_mat* out, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_wgrad(dY, pack, out));
    *bytes = plan_wgrad(dY, pack, out).end;
    return ISO_OK;
}

int32_t iso_act_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out, int32_t accumulate,
                      void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    ISO_TRY(check_wgrad(dY, pack, out));
    if (accumulate != 0 && accumulate != 1) return ISO_ERR_ARG;
    if (share_bytes(bytes_of(out), bytes_of(dY)) || share_bytes(bytes_of(out), codes_of(pack)) ||
        share_bytes(bytes_of(out), exps_of(pack)))
        return ISO_ERR_ARG;
    const WgradPlan p = plan_wgrad(dY, pack, out);
    if (!workspace || ws_bytes < p.end || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    if ((long long)p.m_tiles * p.n_tiles * p.split > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (out->rows == 0 || out->cols == 0) return ISO_OK;
    const long long T = dY->rows, M = out->rows, N = out->cols;
    char* ws = static_cast<char*>(workspace);
    if (T == 0) {
        if (accumulate) return ISO_OK;
        const size_t es = elem_size(out->dtype);
        return cudaMemset2DAsync(out->data, out->ld * es, 0, N * es, M, s) == cudaSuccess ? ISO_OK : ISO_ERR_CUDA;
    }
    const int pairs = resident_pairs();
    if (pairs <= 0) return ISO_ERR_CUDA;

    const iso_mat xb{ws + p.x_bf16, T, N, p.ldx, ISO_BF16, 0};
    ISO_TRY(iso_act_unpack(pack, &xb, stream));
    const int flat_grid = train_sms() * 8;
    if (!p.dy_direct)
        ISO_TRY(by_dtype(dY->dtype, [&](auto* tp) -> int {
            using E = std::remove_pointer_t<decltype(tp)>;
            TRAIN_LAUNCH((k_wgrad_parts<E><<<flat_grid, 256, 0, s>>>(
                static_cast<const E*>(dY->data), dY->ld, (int)T, (int)M,
                reinterpret_cast<__nv_bfloat16*>(ws + p.dy_parts), p.ldd, T * p.ldd)));
            return ISO_OK;
        }));
    WgradMaps maps;
    ISO_TRY(bf16_map(&maps.b, xb.data, T, N, p.ldx));
    for (int q = 0; q < WG_MAX_PARTS; ++q) {
        const int part = std::min(q, p.n_parts - 1);
        if (p.dy_direct)
            ISO_TRY(bf16_map(&maps.a[q], dY->data, T, M, dY->rows == 1 ? (M + 7) / 8 * 8 : dY->ld));
        else
            ISO_TRY(bf16_map(&maps.a[q], ws + p.dy_parts + (size_t)part * T * p.ldd * 2, T, M, p.ldd));
    }
    WgradArgs g{};
    g.M = (int)M;
    g.N = (int)N;
    g.m_tiles = p.m_tiles;
    g.n_tiles = p.n_tiles;
    g.k_tiles = p.k_tiles;
    g.parts = p.n_parts;
    g.split = p.split;
    g.accumulate = accumulate;
    g.out = out->data;
    g.ldo = out->ld;
    g.out_dtype = out->dtype;
    g.out_vec = rows_aligned(out);
    g.part = p.split > 1 ? reinterpret_cast<float*>(ws + p.parts) : nullptr;
    g.ld_part = p.ld_part;
    g.status = status;
    const int items = p.m_tiles * p.n_tiles * p.split;
    TRAIN_LAUNCH((k_wgrad<<<2 * std::min(items, pairs), WG_THREADS, WG_SMEM, s>>>(maps, g)));
    if (p.split == 1) return ISO_OK;
    return by_dtype(out->dtype, [&](auto* op) -> int {
        using O = std::remove_pointer_t<decltype(op)>;
        const int grid = (int)std::min((M * ((N + 7) / 8) + 255) / 256, (long long)flat_grid);
        if (g.out_vec)
            TRAIN_LAUNCH((k_wgrad_join<O, true><<<grid, 256, 0, s>>>(g.part, g.ld_part, g.split, g.M, g.N,
                                                                    static_cast<O*>(out->data), out->ld, accumulate)));
        else
            TRAIN_LAUNCH((k_wgrad_join<O, false><<<grid, 256, 0, s>>>(g.part, g.ld_part, g.split, g.M, g.N,
                                                                     static_cast<O*>(out->data), out->ld, accumulate)));
        return ISO_OK;
    });
}

}  // extern "C"
