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
//              significant bits each, hi + mid + lo = dY (from 2^-110 up; a
//              part's own last bit is 2^-133), and G is the sum of the three
//              products; so every product is exact.
//   k_wgrad    a pair of CTAs per 256 x 256 tile of G, 128 tokens per stage
//              (32 KB of each operand per CTA, three stages; six stages of 64
//              tokens have the same bytes in flight and measured 4 % slower,
//              the waits and commits of a stage costing the same), persistent
//              over the tiles.  The tensor cores add sixteen products at a time
//              and cut low bits off: measured, a product of 2^-25 beside a
//              term of 1 counts, one of 2^-26 does not.  So the error of a
//              binary32 G grows in proportion to the chain of products (1.1e-6,
//              4.4e-7 and 2.0e-7 at chains of 4096, 2048 and 1024 tokens of
//              8192 random ones; a plain binary32 product has 3.1e-7), and is
//              largest where one large product comes before many small ones of
//              one sign (1024 of 2^-27 after a 1: 7.6e-6, as a chain of
//              binary32 additions has).  So a chain is 1024 tokens; the epilogue
//              warps add the
//              chains up in registers, 128 sums a thread, rounding to nearest,
//              while the next chain runs in the other of two accumulators in
//              tensor memory (chains of 2048 measured 1 % faster).
//   measured   18944 x 3584 over 8192 tokens (1.11 PFLOP): 571 us, 1.95
//              PFLOP/s, and 11 us before it for the decoding; a bf16 library
//              product of the same operands 559 - 580 us.  The products
//              themselves bound it (tensor pipe 85 % active), then the copies
//              (472 us without products).
//   split      a G of few tiles under many tokens is cut along the tokens as
//              well; the parts are binary32 in the workspace and k_wgrad_join
//              adds them in order.
#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <algorithm>
#include <atomic>

namespace iso {
namespace {

constexpr int WG_BM = 256;                 // rows of G (dY channels) per CTA pair
constexpr int WG_BK = 128;                 // tokens per stage
constexpr int WG_BOX = 64;                 // channels of one copy: 128 bytes, the swizzle's row
constexpr int WG_BOX_BYTES = WG_BOX * WG_BK * 2;
constexpr int WG_A_BYTES = 2 * WG_BOX_BYTES;           // 128 channels of dY: this CTA's half of a stage
constexpr int WG_EPI_WARPS = 8;
constexpr int WG_OUT_BYTES = 32 * 32 * 4;  // an epilogue warp's 32 x 32 block on its way out
// What depends on BN, the columns of G (X channels) per CTA pair
template <int BN>
struct WgTile {
    static constexpr int B_BOXES = BN / 2 / WG_BOX;        // this CTA's half of X
    static constexpr int STAGE_BYTES = WG_A_BYTES + B_BOXES * WG_BOX_BYTES;
    static constexpr int STAGES = BN == 256 ? 3 : 4;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + WG_EPI_WARPS * WG_OUT_BYTES + 256;
    static constexpr int TMEM_COLS = 2 * BN;               // two accumulators
    static constexpr int BLOCKS = BN / 64;                 // 32-column blocks of an epilogue warp: half the columns
    // kind::f16, fp32 accumulator, bf16 A and B, both MN-major, M = 256 over the pair, N = BN
    static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) |
                                      ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(WG_BM >> 4) << 24);
    static_assert(SMEM <= 232448, "shared memory of one CTA");
};
constexpr int WG_THREADS = (WG_EPI_WARPS + 2) * 32;    // epilogue warps, a copy warp, a product warp
constexpr int WG_MAX_PARTS = WGRAD_PARTS;
constexpr int WG_CHAIN = 8;                // steps accumulated in tensor memory before they are added in registers
// the plan's estimates, in clocks: a step of either tile width, an item's start
// and end, a join's launch and its bytes per clock
constexpr long long WG_STEP_256 = 1250, WG_STEP_128 = 860, WG_ITEM = 4000, WG_JOIN = 4000, WG_JOIN_BYTES = 4100;
// Up to WG_FEW tokens and WG_FEW_WORK multiply-adds take k_wgrad_few.  Measured,
// it against k_wgrad with its operands' kernel: 1 token, G 18944 x 3584 f32 40 / 59
// us, 300 x 200 2.7 / 7.9 us; 16 tokens, 3000 x 1000 9.3 / 13.4 us; 8 tokens,
// 18944 x 3584 74 / 59 us; 32 tokens, 3000 x 1000 14.9 / 12.6 us.
constexpr int WG_FEW = 16;
constexpr long long WG_FEW_WORK = 1LL << 28;
constexpr int FEW_TPB = 128, FEW_WARPS = FEW_TPB / 32, FEW_ROWS = 8;
constexpr int WG_SPLIT_STEPS = 4;          // a part of the tokens has this many steps at least
constexpr int WG_BAND = 8;                 // tile rows that are walked together
constexpr uint64_t WG_WAIT_NS = 2000000000;    // a wait gives up after this long, unless told otherwise
std::atomic<uint64_t> g_wait_ns{WG_WAIT_NS};
constexpr uint64_t WG_LAND_NS = 1000000;       // time given to copies in flight after a give-up

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
    int32_t out_copy;      // blocks leave by bulk copies (maps.out): rows so aligned, nothing to add to
    int32_t* status;
    uint64_t wait_ns;      // limit of a wait for copies, products or accumulators
};
struct WgradMaps {
    CUtensorMap a[WG_MAX_PARTS], b;
    CUtensorMap out;       // G, or the parts of the contraction: columns, rows, part
};

// Shared-memory descriptor of an MN-major operand in the 128-byte swizzle:
// 64 channels (128 bytes) by eight tokens make an atom of 1024 bytes; the next
// eight tokens follow it, the next 64 channels are one copy box further on.
// The start address (in 16-byte words) is the low word's low half, so an
// operand further on in shared memory is an addition to the low word.
constexpr uint32_t WG_DESC_LO = (uint32_t)(WG_BOX_BYTES >> 4) << 16;                    // leading offset: 64 channels on
constexpr uint32_t WG_DESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;                     // stride offset: eight tokens on
__device__ __forceinline__ uint32_t mn_desc_lo(uint32_t saddr) { return WG_DESC_LO + (saddr >> 4); }

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
template <uint32_t IDESC>
__device__ __forceinline__ void umma_bf16_pair(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n\t}"
                 :: "r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(WG_DESC_HI), "r"(IDESC), "r"(accumulate) : "memory");
}
// arrive on this barrier in both CTAs once the products issued so far are done
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"((uint16_t)3) : "memory");
}
// the same, on a barrier of this CTA alone
__device__ __forceinline__ void umma_commit_here(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
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
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Bounded wait: false after limit_ns, or MBAR_SPIN_LIMIT probes.  The probe
// without a time hint measured 2 % faster on the whole product than with one;
// it may suspend the thread for a time of the hardware's choosing, so the
// bound is on the clock as well (WaitClock).
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, uint64_t limit_ns, volatile int* abort_flag) {
    WaitClock clock;
    for (int spin = 0; spin < MBAR_SPIN_LIMIT; ++spin) {
        if (try_wait_cluster(bar, parity)) return true;
        if ((spin & 31) == 31 && (clock.look(now_ns(), limit_ns) || (abort_flag && *abort_flag))) return false;
    }
    return false;
}
// false once the limit is reached or another thread of the CTA gave up, which
// then holds for the whole CTA
__device__ __forceinline__ bool wait_pair(uint32_t bar, uint32_t parity, uint64_t limit_ns, volatile int* abort_flag) {
    if (wait_for(bar, parity, limit_ns, abort_flag)) return true;
    *abort_flag = 1;
    return false;
}
// 16 consecutive columns of this thread's accumulator row; the values may be
// used after the wait below, which takes them as operands so that no use is
// moved before it
__device__ __forceinline__ void tmem_load(uint32_t taddr, float (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
                   "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]),
                   "=f"(v[14]), "=f"(v[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(float (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]),
                   "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]),
                   "+f"(v[14]), "+f"(v[15])
                 :: "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A warp's 32 x 32 block of G: lane l holds row l.  Into shared memory, rows of
// 128 bytes, their 16-byte words swizzled by row (no bank is hit twice, and a
// bulk copy with the 128-byte swizzle reads it).
__device__ __forceinline__ void stage_block(float4* buf, const float (&v)[32], int lane) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        buf[lane * 8 + (j ^ (lane & 7))] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
// The staged block to G where bulk copies cannot: a store covers whole runs of
// a row, 16-byte words of eight (f32) or four (bf16) lanes where G's rows
// start on 16-byte boundaries, else a row's 32 columns by the 32 lanes.
template <typename O>
__device__ __forceinline__ void store_block(const float4* buf, int lane, O* out, long long ldo, int m, int n, int M, int N,
                                         bool vec, int accumulate) {
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

// The warp's block out of shared memory by a bulk copy, clipped at G's edges.
// G itself is not read again soon and leaves L2 first (200 tokens, 8960 x 8960
// f32: 77 -> 70 us); the parts of a split are.
__device__ __forceinline__ void copy_out(const CUtensorMap* map, uint32_t src, int n, int m, int part, bool keep) {
    uint64_t policy;
    if (keep) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group.L2::cache_hint [%0, {%1, %2, %3}], [%4], %5;"
                 :: "l"(reinterpret_cast<uint64_t>(map)), "r"(n), "r"(m), "r"(part), "r"(src), "l"(policy) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// the buffer of the copies so far may be written again
__device__ __forceinline__ void copies_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Work item i: a part of the contraction of one tile; tiles in bands of
// WG_BAND tile rows, column by column inside a band, so that the pairs that
// run together share their operands' rows in L2.
template <int BN>
__device__ __forceinline__ void work_item(const WgradArgs& g, int i, int& m0, int& n0, int& k0, int& k1, int& part) {
    const int tile = i / g.split;
    part = i - tile * g.split;
    const int band = tile / (WG_BAND * g.n_tiles), in = tile - band * WG_BAND * g.n_tiles;
    const int rows = min(WG_BAND, g.m_tiles - band * WG_BAND);
    m0 = (band * WG_BAND + in % rows) * WG_BM;
    n0 = in / rows * BN;
    k0 = (int)((long long)g.k_tiles * part / g.split);
    k1 = (int)((long long)g.k_tiles * (part + 1) / g.split);
}

template <int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WG_THREADS, 1)
k_wgrad(const __grid_constant__ WgradMaps maps, WgradArgs g) {
    using Tile = WgTile<BN>;
    constexpr int STAGES = Tile::STAGES, STAGE_BYTES = Tile::STAGE_BYTES;
    extern __shared__ unsigned char wg_smem_raw[];
    unsigned char* const smem =
        reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(wg_smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* const bars =
        reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES + WG_EPI_WARPS * WG_OUT_BYTES);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 5);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const uint32_t st = smem_u32(smem), bar = smem_u32(bars);
    auto full = [&](int s) { return bar + 8u * s; };                          // leader: both CTAs' copies landed
    auto empty = [&](int s) { return bar + 8u * (STAGES + s); };           // products that read the stage are done
    auto acc_full = [&](int a) { return bar + 8u * (2 * STAGES + a); };    // accumulator complete
    auto acc_empty = [&](int a) { return bar + 8u * (2 * STAGES + 2 + a); };   // leader: accumulator read by all
    const uint32_t all_done = bar + 8u * (2 * STAGES + 4);                     // leader: every product issued is done

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(acc_full(a), 1);
            mbar_init(acc_empty(a), 2 * WG_EPI_WARPS);
        }
        mbar_init(all_done, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_u32(tmem_slot)), "r"(Tile::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_barrier();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
    start_next();
    wait_before();           // the operands are written by the kernel before
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int items = g.m_tiles * g.n_tiles * g.split;

    if (warp == WG_EPI_WARPS && lane == 0) {
        // copies: this CTA's 128 channels of either operand
        const uint32_t full0 = in_leader(full(0));
        uint32_t s = 0, ph = 1, done = 0;            // stage, its parity, copies issued
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item<BN>(g, i, m0, n0, k0, k1, part);
            m0 += (int)rank * 128;
            n0 += (int)rank * (BN / 2);
            int p = k0 / g.t_tiles, t = (k0 - p * g.t_tiles) * WG_BK;
            for (int k = k0; k < k1; ++k) {
                if (!wait_pair(empty(s), ph, g.wait_ns, abort_flag)) { ok = false; break; }
                if (rank == 0) mbar_arrive_tx(full(s), 2 * STAGE_BYTES);
                const CUtensorMap* am = &maps.a[p];
                const uint32_t fb = full0 + 8u * s, a = st + s * STAGE_BYTES, b = a + WG_A_BYTES;
                tma_load_pair(a, am, m0, t, fb);
                tma_load_pair(a + WG_BOX_BYTES, am, m0 + WG_BOX, t, fb);
#pragma unroll
                for (int q = 0; q < Tile::B_BOXES; ++q)
                    tma_load_pair(b + q * WG_BOX_BYTES, &maps.b, n0 + q * WG_BOX, t, fb);
                if ((t += WG_BK) >= g.t_tiles * WG_BK) { t = 0; ++p; }
                if (++s == STAGES) { s = 0; ph ^= 1u; }
                ++done;
            }
        }
        // every copy into this CTA has been consumed before it may exit: the
        // products that read a stage free it in both CTAs.  After a give-up the
        // products may not come; the waits then let the copies land, which takes
        // microseconds.
        for (uint32_t q = 0; q < min(done, (uint32_t)STAGES); ++q) {
            if (s == 0) { s = STAGES; ph ^= 1u; }
            --s;
            if (!wait_for(empty(s), ph ^ 1u, WG_WAIT_NS, abort_flag)) wait_for(empty(s), ph ^ 1u, WG_LAND_NS, nullptr);
        }
    } else if (warp == WG_EPI_WARPS + 1 && lane == 0 && rank == 0) {
        // products of the pair, chain by chain
        const uint32_t a0 = mn_desc_lo(st), b0 = mn_desc_lo(st + WG_A_BYTES);
        uint32_t s = 0, ph = 0, acc = 0, acc_ph = 1;
        bool ok = true;
        for (int i = pair; ok && i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item<BN>(g, i, m0, n0, k0, k1, part);
            for (int kc = k0; ok && kc < k1; kc += WG_CHAIN) {
                if (!wait_pair(acc_empty(acc), acc_ph, g.wait_ns, abort_flag)) { ok = false; break; }
                tc_after();
                const uint32_t d = tmem + acc * BN;
                uint32_t more = 0;
                for (int k = min(k1 - kc, WG_CHAIN); k > 0; --k) {
                    if (!wait_pair(full(s), ph, g.wait_ns, abort_flag)) { ok = false; break; }
                    tc_after();
                    const uint32_t a = a0 + s * (STAGE_BYTES >> 4), b = b0 + s * (STAGE_BYTES >> 4);
#pragma unroll
                    for (uint32_t q = 0; q < WG_BK / 16; ++q) {   // 16 tokens per product: two atoms of eight
                        umma_bf16_pair<Tile::IDESC>(d, a + (2048u >> 4) * q, b + (2048u >> 4) * q, more);
                        more = 1;
                    }
                    umma_commit_pair(empty(s));
                    if (++s == STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;                       // the accumulator is not complete
                umma_commit_pair(acc_full(acc));
                acc ^= 1u;
                if (acc == 0) acc_ph ^= 1u;
            }
        }
        // no product runs on when the tensor memory is freed, after a give-up either
        umma_commit_here(all_done);
        wait_for(all_done, 0, WG_WAIT_NS, nullptr);
    } else if (warp < WG_EPI_WARPS) {
        // epilogue: warp w reads tensor-memory lanes 32 (w mod 4) ..., half of the columns
        const int quad = warp & 3, half = warp >> 2;
        float4* const buf = reinterpret_cast<float4*>(smem + STAGES * STAGE_BYTES + warp * WG_OUT_BYTES);
        int n_acc = 0;
        bool ok = true;
        for (int i = pair; i < items; i += pairs) {
            int m0, n0, k0, k1, part;
            work_item<BN>(g, i, m0, n0, k0, k1, part);
            float sum[Tile::BLOCKS][32];
#pragma unroll
            for (int c = 0; c < Tile::BLOCKS; ++c)
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[c][j] = 0.0f;
            for (int kc = k0; ok && kc < k1; kc += WG_CHAIN, ++n_acc) {
                const int acc = n_acc & 1;
                // one answer for the warp: loads of tensor memory take all of its lanes
                ok = __all_sync(0xFFFFFFFFu, wait_pair(acc_full(acc), (uint32_t)(n_acc >> 1) & 1u, g.wait_ns, abort_flag));
                if (!ok) break;
                tc_after();
                const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * BN + half * (BN / 2));
                // 16 columns at a time: reading a chain's block in one go holds the next chain's
                // products up (730 us against 590 for 18944 x 3584 over 8192 tokens)
#pragma unroll
                for (int c = 0; c < 2 * Tile::BLOCKS; ++c) {
                    float v[16];
                    tmem_load(at + c * 16, v);
                    tmem_wait(v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c >> 1][(c & 1) * 16 + j] += v[j];
                }
                tc_before();
                __syncwarp();
                if (lane == 0) arrive_cluster(in_leader(acc_empty(acc)));
            }
            if (!ok) {       // blocks that a give-up left without their sums are NaN
#pragma unroll
                for (int c = 0; c < Tile::BLOCKS; ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[c][j] = __int_as_float(0x7FFFFFFF);
            }
            const int m = m0 + (int)rank * 128 + quad * 32;
            if (m >= g.M) continue;
            if (g.out_copy) {
                // 32 rows of 128 bytes, their 16-byte words swizzled by row as the copy expects them
                const bool narrow = g.split == 1 && g.out_dtype == ISO_BF16;
#pragma unroll
                for (int c = 0; c < Tile::BLOCKS; ++c) {
                    const int n = n0 + half * (BN / 2) + c * 32;
                    if (!narrow || (c & 1) == 0) {
                        if (lane == 0) copies_read();
                        __syncwarp();
                    }
                    if (narrow) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            reinterpret_cast<uint4*>(buf)[lane * 8 + (((c & 1) * 4 + j) ^ (lane & 7))] =
                                make_uint4(f32_to_bf16x2(sum[c][8 * j], sum[c][8 * j + 1]),
                                           f32_to_bf16x2(sum[c][8 * j + 2], sum[c][8 * j + 3]),
                                           f32_to_bf16x2(sum[c][8 * j + 4], sum[c][8 * j + 5]),
                                           f32_to_bf16x2(sum[c][8 * j + 6], sum[c][8 * j + 7]));
                    } else {
                        stage_block(buf, sum[c], lane);
                    }
                    if (!narrow || (c & 1) == 1) {
                        const int first = narrow ? n - 32 : n;
                        fence_async_shared();
                        __syncwarp();
                        if (lane == 0 && first < g.N) copy_out(&maps.out, smem_u32(buf), first, m, part, g.split > 1);
                    }
                }
                continue;
            }
#pragma unroll
            for (int c = 0; c < Tile::BLOCKS; ++c) {
                const int n = n0 + half * (BN / 2) + c * 32;
                __syncwarp();
                stage_block(buf, sum[c], lane);
                __syncwarp();
                if (n >= g.N) continue;
                if (g.out_dtype == ISO_BF16)
                    store_block(buf, lane, static_cast<__nv_bfloat16*>(g.out), g.ldo, m, n, g.M, g.N, g.out_vec,
                                g.accumulate);
                else
                    store_block(buf, lane, static_cast<float*>(g.out), g.ldo, m, n, g.M, g.N, g.out_vec, g.accumulate);
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    cluster_barrier();       // neither CTA exits while the other's products or arrivals may touch it
    if (threadIdx.x == 0 && *abort_flag && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_TIMEOUT);
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(Tile::TMEM_COLS) : "memory");
    }
}

// Few tokens: the tensor cores' fixed costs (the operands' kernel, a step of 128
// tokens, the accumulator's way out) outweigh the products.  Here a warp holds
// FEW_ROWS x 256 of G in registers and adds token by token, decoding X on the
// way; dY's values of the block are staged in shared memory.
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(FEW_TPB) k_wgrad_few(const T* dy, long long ldd, const uint8_t* codes, long long ldc,
                                                       const uint8_t* exps, long long lde, O* out, long long ldo,
                                                       int tokens, int M, int N, int m_blocks, int accumulate) {
    constexpr int ROWS = FEW_WARPS * FEW_ROWS;
    __shared__ __align__(16) float d[WG_FEW][ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nb = blockIdx.x / m_blocks, mb = blockIdx.x - nb * m_blocks;
    const int c = nb * TRAIN_SEG + lane * 8;
    for (int i = threadIdx.x; i < tokens * ROWS; i += FEW_TPB) {
        const int t = i / ROWS, m = mb * ROWS + i % ROWS;
        d[t][i % ROWS] = m < M ? to_f32(dy[t * ldd + m]) : 0.0f;
    }
    __syncthreads();
    float acc[FEW_ROWS][8] = {};
#pragma unroll 2
    for (int t = 0; t < tokens; ++t) {
        uint2 q = make_uint2(0u, 0u);
        uint32_t b = 1;
        if (c < N) {   // codes are padded to whole groups of 32 channels
            q = *reinterpret_cast<const uint2*>(codes + t * ldc + c);
            b = exps[t * lde + c / ISO_ACT_GROUP];
        }
        float x[8];
        act_decode(q, b, x);
#pragma unroll
        for (int r = 0; r < FEW_ROWS; r += 4) {
            const float4 w = *reinterpret_cast<const float4*>(&d[t][warp * FEW_ROWS + r]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[r][j] = fmaf(w.x, x[j], acc[r][j]);
                acc[r + 1][j] = fmaf(w.y, x[j], acc[r + 1][j]);
                acc[r + 2][j] = fmaf(w.z, x[j], acc[r + 2][j]);
                acc[r + 3][j] = fmaf(w.w, x[j], acc[r + 3][j]);
            }
        }
    }
    const int m0 = mb * ROWS + warp * FEW_ROWS;
    if (c >= N) return;
#pragma unroll
    for (int r = 0; r < FEW_ROWS; ++r) {
        if (m0 + r >= M) break;
        O* row = out + (long long)(m0 + r) * ldo;
        if (accumulate) {
            float old[8];
            load8<VEC>(row, c, N, old);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[r][j] += old[j];
        }
        if (VEC && c + 8 <= N) put8(row + c, acc[r]);
        else store8<false>(row, c, N, acc[r]);
    }
}

// out (+)= the sum of the parts in order
template <typename O, bool VEC>
__global__ void __launch_bounds__(256) k_wgrad_join(const float* part, long long ld_part, int split, int M, int N,
                                                    O* out, long long ldo, int accumulate) {
    wait_before();
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

// G or its parts: cols, rows, parts; blocks of 32 rows of 128 bytes
int out_map(CUtensorMap* map, void* base, int32_t dtype, long long rows, long long cols, long long ld, int parts) {
    EncodeTiled fn = encode_tiled();
    if (!fn) return ISO_ERR_CUDA;
    const long long es = elem_size(dtype);
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts};
    const cuuint64_t strides[2] = {(cuuint64_t)(ld * es), (cuuint64_t)(rows * ld * es)};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / es), 32, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, dtype == ISO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims,
              strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
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
template <int BN>
int resident_pairs() {
    static std::atomic<int> pairs[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = pairs[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaFuncSetAttribute(k_wgrad<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, WgTile<BN>::SMEM) != cudaSuccess)
            return 0;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(train_sms() / 2 * 2));
        cfg.blockDim = dim3(WG_THREADS);
        cfg.dynamicSmemBytes = WgTile<BN>::SMEM;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 2;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, k_wgrad<BN>, &cfg) != cudaSuccess || n <= 0) return 0;
        pairs[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// The product; it may be set up while the operands' kernel ends, and waits for it.
template <int BN>
int launch_wgrad(const WgradMaps& maps, const WgradArgs& g, int items, cudaStream_t s) {
    const int pairs = resident_pairs<BN>();
    if (pairs <= 0) return ISO_ERR_CUDA;
    TRAIN_LAUNCH(launch_early(k_wgrad<BN>, (unsigned)(2 * std::min(items, pairs)), WG_THREADS, WgTile<BN>::SMEM, s, maps, g));
    return ISO_OK;
}

bool few_tokens(long long T, long long M, long long N) {
    return T <= WG_FEW && (long double)T * M * N <= (long double)WG_FEW_WORK;
}

struct WgradPlan {
    size_t x_bf16, dy_parts, parts, end;
    long long ldx, ldd, ld_part;
    int bn, m_tiles, n_tiles, k_tiles, split, n_parts;
    bool dy_direct;
};
// Host only, the same for the sizing call and the launch (the pair count of a
// GB300 stands in where there is no device).
WgradPlan plan_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out) {
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    WgradPlan p{};
    const long long T = dY->rows, M = out->rows, N = out->cols;
    if (few_tokens(T, M, N)) {
        p.end = 256;
        return p;
    }
    p.n_parts = dY->dtype == ISO_F32 ? 3 : 1;
    p.dy_direct = dY->dtype == ISO_BF16 && (reinterpret_cast<uintptr_t>(dY->data) & 15u) == 0 && dY->ld % 8 == 0;
    p.m_tiles = (int)((M + WG_BM - 1) / WG_BM);
    p.k_tiles = (int)((T + WG_BK - 1) / WG_BK) * p.n_parts;
    // Tile width and token split by the estimated time of the longest-running
    // pair, in clocks
    const long long pairs = std::max(1, train_sms() / 2);
    long long best = -1;
    for (int bn : {256, 128}) {
        const long long n_tiles = (N + bn - 1) / bn, tiles = p.m_tiles * n_tiles;
        for (int split : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (split > 1 && p.k_tiles / split < WG_SPLIT_STEPS) break;
            const long long rounds = (tiles * split + pairs - 1) / pairs, steps = (p.k_tiles + split - 1) / split;
            const long long cost = rounds * (steps * (bn == 256 ? WG_STEP_256 : WG_STEP_128) + WG_ITEM) +
                                   (split > 1 ? WG_JOIN + M * N * (split + 1) * 4 / WG_JOIN_BYTES : 0);
            if (best < 0 || cost < best) {
                best = cost;
                p.bn = bn;
                p.n_tiles = (int)n_tiles;
                p.split = split;
            }
        }
    }
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

int64_t iso_act_wgrad_wait_ns(int64_t ns) {
    return (int64_t)(ns < 0 ? g_wait_ns.load(std::memory_order_relaxed)
                            : g_wait_ns.exchange((uint64_t)ns, std::memory_order_relaxed));
}

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
    if (few_tokens(T, M, N)) {
        const long long m_blocks = (M + FEW_WARPS * FEW_ROWS - 1) / (FEW_WARPS * FEW_ROWS), n_blocks = (N + TRAIN_SEG - 1) / TRAIN_SEG;
        if (m_blocks * n_blocks > EXTENT_LIMIT) return ISO_ERR_UNSUPPORTED;
        return by_dtype(dY->dtype, [&](auto* tp) -> int {
            return by_dtype(out->dtype, [&](auto* op) -> int {
                using E = std::remove_pointer_t<decltype(tp)>;
                using O = std::remove_pointer_t<decltype(op)>;
                auto go = [&](auto v) -> int {
                    TRAIN_LAUNCH((k_wgrad_few<E, O, decltype(v)::value><<<(unsigned)(m_blocks * n_blocks), FEW_TPB, 0, s>>>(
                        static_cast<const E*>(dY->data), dY->ld, static_cast<const uint8_t*>(pack->codes), pack->ld_codes,
                        static_cast<const uint8_t*>(pack->exps), pack->ld_exps, static_cast<O*>(out->data), out->ld,
                        (int)T, (int)M, (int)N, (int)m_blocks, accumulate)));
                    return ISO_OK;
                };
                return rows_aligned(out) ? go(std::true_type{}) : go(std::false_type{});
            });
        });
    }

    __nv_bfloat16* const xb = reinterpret_cast<__nv_bfloat16*>(ws + p.x_bf16);
    __nv_bfloat16* const dy_parts = reinterpret_cast<__nv_bfloat16*>(ws + p.dy_parts);
    ISO_TRY(launch_wgrad_operands(pack, xb, p.ldx, p.dy_direct ? nullptr : dY, dy_parts, p.ldd, s));
    WgradMaps maps;
    ISO_TRY(bf16_map(&maps.b, xb, T, N, p.ldx));
    for (int q = 0; q < p.n_parts; ++q) {
        const int part = p.n_parts - 1 - q;      // the last part first: small sums before large ones
        if (p.dy_direct)
            ISO_TRY(bf16_map(&maps.a[q], dY->data, T, M, dY->ld));
        else
            ISO_TRY(bf16_map(&maps.a[q], dy_parts + (size_t)part * T * p.ldd, T, M, p.ldd));
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
    // A bulk copy's rows start on 16-byte boundaries and end on them: at the last
    // column it clips whole 16-byte words only, and what stands beside G in a
    // wider buffer is not the call's to write.  (The parts' rows are padded.)
    const int es = elem_size(out->dtype);
    g.out_copy = p.split > 1 || (!accumulate && g.out_vec && (out->ld * es) % 16 == 0 && (N * es) % 16 == 0);
    float* const parts = reinterpret_cast<float*>(ws + p.parts);
    if (p.split > 1)
        ISO_TRY(out_map(&maps.out, parts, ISO_F32, M, N, p.ld_part, p.split));
    else if (g.out_copy)
        ISO_TRY(out_map(&maps.out, out->data, out->dtype, M, N, out->ld, 1));
    g.status = status;
    g.wait_ns = g_wait_ns.load(std::memory_order_relaxed);
    const int items = p.m_tiles * p.n_tiles * p.split;
    ISO_TRY(p.bn == 256 ? launch_wgrad<256>(maps, g, items, s) : launch_wgrad<128>(maps, g, items, s));
    if (p.split == 1) return ISO_OK;
    return by_dtype(out->dtype, [&](auto* op) -> int {
        using O = std::remove_pointer_t<decltype(op)>;
        const int grid = (int)std::min((M * ((N + 7) / 8) + 255) / 256, (long long)EXTENT_LIMIT);
        TRAIN_LAUNCH(launch_early(g.out_vec ? k_wgrad_join<O, true> : k_wgrad_join<O, false>, (unsigned)grid, 256u, 0, s,
                                  parts, p.ld_part, g.split, g.M, g.N, static_cast<O*>(out->data), out->ld, accumulate));
        return ISO_OK;
    });
}

}  // extern "C"
