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
//   k_wgrad    a pair of CTAs per 256 x 256 tile of G, 128 tokens per stage
//              (32 KB of each operand per CTA, three stages; six stages of 64
//              tokens have the same bytes in flight and measured 4 % slower,
//              the waits and commits of a stage costing the same), persistent
//              over the tiles.  The tensor cores' accumulation cuts low bits
//              off at every product: the relative error of a binary32 G grows
//              in proportion to the chain of products (1.1e-6, 4.4e-7 and 2.0e-7 at chains of 4096, 2048 and 1024
//              tokens of 8192 random ones; a plain binary32 product has
//              3.1e-7).  So a chain is 1024 tokens; the epilogue warps add the
//              chains up in registers, 128 sums a thread, rounding to nearest,
//              while the next chain runs in the other of two accumulators in
//              tensor memory (chains of 2048 measured 1 % faster).
//   measured   18944 x 3584 over 8192 tokens (1.11 PFLOP): 579 us alone, 1922
//              TFLOP/s, with 16 us before it for the decoding; a bf16 library
//              product of the same operands 559 - 580 us.  The products
//              themselves bound it, then the copies (about 470 us alone).
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
constexpr int WG_BK = 128;                 // tokens per stage
constexpr int WG_STAGES = 3;
constexpr int WG_BOX = 64;                 // channels of one copy: 128 bytes, the swizzle's row
constexpr int WG_BOX_BYTES = WG_BOX * WG_BK * 2;
constexpr int WG_OP_BYTES = 2 * WG_BOX_BYTES;          // 128 channels of an operand: this CTA's half
constexpr int WG_STAGE_BYTES = 2 * WG_OP_BYTES;
constexpr int WG_EPI_WARPS = 8;
constexpr int WG_OUT_BYTES = 32 * 32 * 4;  // an epilogue warp's 32 x 32 block on its way out
constexpr int WG_SMEM = 1024 + WG_STAGES * WG_STAGE_BYTES + WG_EPI_WARPS * WG_OUT_BYTES + 256;
static_assert(WG_SMEM <= 232448, "shared memory of one CTA");
constexpr int WG_THREADS = (WG_EPI_WARPS + 2) * 32;    // epilogue warps, a copy warp, a product warp
constexpr int WG_MAX_PARTS = 3;
constexpr int WG_MAX_SPLIT = 8;
constexpr int WG_CHAIN = 8;                // steps accumulated in tensor memory before they are added in registers
constexpr int WG_BAND = 8;                 // tile rows that are walked together

struct WgradArgs {
    int32_t M, N;
    int32_t m_tiles, n_tiles;
    int32_t t_tiles;       // steps over the tokens: ceil(tokens / 128)
    int32_t k_tiles;       // steps of the whole contraction: parts x t_tiles, part after part
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
// The start address (in 16-byte words) is the low word's low half, so an
// operand further on in shared memory is an addition to the low word.
constexpr uint32_t WG_DESC_LO = (uint32_t)(WG_BOX_BYTES >> 4) << 16;                    // leading offset: 64 channels on
constexpr uint32_t WG_DESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;                     // stride offset: eight tokens on
__device__ __forceinline__ uint32_t mn_desc_lo(uint32_t saddr) { return WG_DESC_LO + (saddr >> 4); }

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
__device__ __forceinline__ void umma_bf16_pair(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n\t}"
                 :: "r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(WG_DESC_HI), "r"(WG_IDESC), "r"(accumulate) : "memory");
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
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
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
// 16 consecutive columns of this thread's accumulator row
__device__ __forceinline__ void tmem_load16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                   "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
                   "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A warp's 32 x 32 block of G: lane l holds row l.  Through shared memory
// (16-byte words swizzled by row), so that a store covers whole runs of a row:
// one row by 16-byte words of eight (f32) or four (bf16) lanes where G's rows
// start on 16-byte boundaries, else a row's 32 columns by the 32 lanes.
template <typename O>
__device__ __forceinline__ void store_block(float4* buf, const float (&v)[32], int lane, O* out, long long ldo, int m,
                                            int n, int M, int N, bool vec, int accumulate) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)
        buf[lane * 8 + (j ^ (lane & 7))] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    __syncwarp();
    const int rows = min(32, M - m);
    if (vec && n + 32 <= N) {
        if constexpr (sizeof(O) == 4) {
#pragma unroll 2
            for (int i = 0; i < 8; ++i) {
                const int r = i * 4 + (lane >> 3), w = lane & 7;
                if (r >= rows) continue;
                float4 x = buf[r * 8 + (w ^ (r & 7))];
                float4* o = reinterpret_cast<float4*>(out + (long long)(m + r) * ldo + n) + w;
                if (accumulate) {
                    const float4 old = *o;
                    x.x += old.x; x.y += old.y; x.z += old.z; x.w += old.w;
                }
                *o = x;
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2), w = (lane & 3) * 2;
                if (r >= rows) continue;
                const float4 x = buf[r * 8 + (w ^ (r & 7))], y = buf[r * 8 + ((w + 1) ^ (r & 7))];
                float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                O* o = out + (long long)(m + r) * ldo;
                if (accumulate) {
                    float old[8];
                    load8<true>(o, n + w * 4, N, old);
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] += old[k];
                }
                store8<true>(o, n + w * 4, N, f);
            }
        }
    } else if (n + lane < N) {
        const float* flat = reinterpret_cast<const float*>(buf);
#pragma unroll 1
        for (int r = 0; r < rows; ++r) {
            const float x = flat[r * 32 + (((lane >> 2) ^ (r & 7)) << 2) + (lane & 3)];
            O* o = out + (long long)(m + r) * ldo + n + lane;
            from_f32(accumulate ? to_f32(*o) + x : x, *o);
        }
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
    uint64_t* const bars =
        reinterpret_cast<uint64_t*>(smem + WG_STAGES * WG_STAGE_BYTES + WG_EPI_WARPS * WG_OUT_BYTES);
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
        const uint32_t full0 = in_leader(full(0)), own = rank * 128;
        uint32_t s = 0, ph = 1, done = 0;            // stage, its parity, copies issued
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            m0 += own;
            n0 += own;
            int p = k0 / g.t_tiles, t = (k0 - p * g.t_tiles) * WG_BK;
            for (int k = k0; k < k1; ++k) {
                if (!wait_pair(empty(s), ph, abort_flag)) { ok = false; break; }
                if (rank == 0) mbar_arrive_tx(full(s), 2 * WG_STAGE_BYTES);
                const CUtensorMap* am = &maps.a[p];
                const uint32_t fb = full0 + 8u * s, a = st + s * WG_STAGE_BYTES, b = a + WG_OP_BYTES;
                tma_load_pair(a, am, m0, t, fb);
                tma_load_pair(a + WG_BOX_BYTES, am, m0 + WG_BOX, t, fb);
                tma_load_pair(b, &maps.b, n0, t, fb);
                tma_load_pair(b + WG_BOX_BYTES, &maps.b, n0 + WG_BOX, t, fb);
                if ((t += WG_BK) >= g.t_tiles * WG_BK) { t = 0; ++p; }
                if (++s == WG_STAGES) { s = 0; ph ^= 1u; }
                ++done;
            }
        }
        // every copy into this CTA has been consumed before it may exit: the
        // products that read a stage free it in both CTAs
        for (uint32_t q = 0; q < min(done, (uint32_t)WG_STAGES); ++q) {
            if (s == 0) { s = WG_STAGES; ph ^= 1u; }
            --s;
            for (int spin = 0; spin < MBAR_SPIN_LIMIT; ++spin)
                if (try_wait_cluster(empty(s), ph ^ 1u) || *abort_flag) break;
        }
    } else if (warp == WG_EPI_WARPS + 1 && lane == 0 && rank == 0) {
        // products of the pair, chain by chain
        const uint32_t a0 = mn_desc_lo(st), b0 = mn_desc_lo(st + WG_OP_BYTES);
        uint32_t s = 0, ph = 0, acc = 0, acc_ph = 1;
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            for (int kc = k0; ok && kc < k1; kc += WG_CHAIN) {
                if (!wait_pair(acc_empty(acc), acc_ph, abort_flag)) { ok = false; break; }
                tc_after();
                const uint32_t d = tmem + acc * WG_BN;
                uint32_t more = 0;
                for (int k = min(k1 - kc, WG_CHAIN); k > 0; --k) {
                    if (!wait_pair(full(s), ph, abort_flag)) { ok = false; break; }
                    tc_after();
                    const uint32_t a = a0 + s * (WG_STAGE_BYTES >> 4), b = b0 + s * (WG_STAGE_BYTES >> 4);
#pragma unroll
                    for (uint32_t q = 0; q < WG_BK / 16; ++q) {   // 16 tokens per product: two atoms of eight
                        umma_bf16_pair(d, a + (2048u >> 4) * q, b + (2048u >> 4) * q, more);
                        more = 1;
                    }
                    umma_commit_pair(empty(s));
                    if (++s == WG_STAGES) { s = 0; ph ^= 1u; }
                }
                umma_commit_pair(acc_full(acc));
                acc ^= 1u;
                if (acc == 0) acc_ph ^= 1u;
            }
        }
    } else if (warp < WG_EPI_WARPS) {
        // epilogue: warp w reads tensor-memory lanes 32 (w mod 4) ..., 128 of the 256 columns
        const int quad = warp & 3, half = warp >> 2;
        float4* const buf = reinterpret_cast<float4*>(smem + WG_STAGES * WG_STAGE_BYTES + warp * WG_OUT_BYTES);
        int n_acc = 0;
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item(g, i, m0, n0, k0, k1, part);
            float sum[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[c][j] = 0.0f;
            for (int kc = k0; kc < k1; kc += WG_CHAIN, ++n_acc) {
                const int acc = n_acc & 1;
                if (!wait_pair(acc_full(acc), (uint32_t)(n_acc >> 1) & 1u, abort_flag)) { ok = false; break; }
                __syncwarp();
                tc_after();
                const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * WG_BN + half * 128);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float v[16];
                    tmem_load16(at + c * 16, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c >> 1][(c & 1) * 16 + j] += v[j];
                }
                tc_before();
                __syncwarp();
                if (lane == 0) arrive_cluster(in_leader(acc_empty(acc)));
            }
            if (!ok) break;
            const int m = m0 + (int)rank * 128 + quad * 32;
            if (m >= g.M) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int n = n0 + half * 128 + c * 32;
                if (n >= g.N) continue;
                if (g.part)
                    store_block(buf, sum[c], lane, g.part + (long long)part * g.M * g.ld_part, g.ld_part, m, n, g.M,
                                g.N, true, 0);
                else if (g.out_dtype == ISO_BF16)
                    store_block(buf, sum[c], lane, static_cast<__nv_bfloat16*>(g.out), g.ldo, m, n, g.M, g.N,
                                g.out_vec, g.accumulate);
                else
                    store_block(buf, sum[c], lane, static_cast<float*>(g.out), g.ldo, m, n, g.M, g.N, g.out_vec,
                                g.accumulate);
            }
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
    // cut the tokens where the tiles leave half the pairs idle, four steps a part at least
    p.split = (int)std::max(1LL, std::min({pairs / std::max(1LL, tiles), (long long)p.k_tiles / 4, (long long)WG_MAX_SPLIT}));
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
        const int part = std::max(0, p.n_parts - 1 - q);     // the last part first: small sums before large ones
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
    g.t_tiles = p.k_tiles / p.n_parts;
    g.k_tiles = p.k_tiles;
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
