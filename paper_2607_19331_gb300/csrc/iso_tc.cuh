// iso_tc.cuh -- the fifth-generation tensor cores as the attention kernels use
// them (one CTA per product): tiles of 128 rows by tensor copies, bf16 products
// with their accumulator (and a bf16 A operand) in tensor memory, bounded waits.
#pragma once

#include <cuda.h>

#include "iso_train.cuh"
#include "iso_internal.cuh"

namespace iso {
namespace tc {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int ROWS = 128;                      // rows of a tile
constexpr int BOX = 64;                        // channels of one copy: 128 bytes, the swizzle's row
constexpr int BOX_BYTES = ROWS * BOX * 2;

// kind::f16, fp32 accumulator, bf16 operands, M = 128, N = n; b_rows: B's
// contraction runs over its rows ("MN-major") instead of along them
constexpr uint32_t idesc(int n, bool b_rows) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_rows ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(ROWS >> 4) << 24);
}
// Shared-memory descriptors of a tile in the 128-byte swizzle (atoms of eight
// rows, 1024 bytes): the high word for both, the low word is the start address in
// 16-byte words and, where the contraction runs over rows, the distance of the
// next 64 channels.
constexpr uint32_t DESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;
constexpr uint32_t DESC_LO_ALONG = 1u << 16, DESC_LO_ROWS = (uint32_t)(BOX_BYTES >> 4) << 16;

// D (+)= A B^T, A and B tiles in shared memory, contraction along their rows
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t desc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
                 :: "r"(d), "r"(a_lo), "r"(b_lo), "r"(DESC_HI), "r"(desc), "r"(accumulate) : "memory");
}
// D (+)= A B, A in tensor memory (two bf16 a column, the lower half first)
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t desc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "mov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
                 :: "r"(d), "r"(a), "r"(b_lo), "r"(DESC_HI), "r"(desc), "r"(accumulate) : "memory");
}
// D = A B^T over DP channels: two tiles of 128 rows (DP / 64 boxes each)
template <int DP>
__device__ __forceinline__ void product_along(uint32_t d, uint32_t a, uint32_t b) {
    const uint32_t al = DESC_LO_ALONG + (a >> 4), bl = DESC_LO_ALONG + (b >> 4);
#pragma unroll
    for (uint32_t k = 0; k < DP / 16; ++k) {
        const uint32_t at = (k / 4) * (BOX_BYTES >> 4) + (k % 4) * 2;
        mma_ss(d, al + at, bl + at, idesc(ROWS, false), k > 0);
    }
}
// D (+)= A B: A [128 x 128] bf16 in tensor memory, each COLS columns of it (COLS / 2
// words) at the place of as many binary32 ones; B the tile's 128 rows of DP channels
template <int DP, int COLS>
__device__ __forceinline__ void product_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t accumulate) {
    const uint32_t bl = DESC_LO_ROWS + (b >> 4);
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
        mma_ts(d, a + k * 16 / COLS * COLS + k * 16 % COLS / 2, bl + k * (2048u >> 4), idesc(DP, true), k > 0 ? 1u : accumulate);
}

// One lane of the warp, the same each time, as the hardware elects it: code under
// it keeps its descriptors in uniform registers, where a branch on the lane's number
// moves each there for every product (8192 tokens, 28 heads of 128: dk and dv
// 935 -> 810 us).  Called by the whole warp.
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// A slot of a ring of copies and the parity of its next phase
template <int N>
struct Slot {
    int at = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            parity ^= 1u;
        }
    }
};

// arrive on `bar` once the products issued so far are done
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 consecutive words of this thread's row of tensor memory; usable after the
// wait, which takes them as operands so that no use is moved before it
__device__ __forceinline__ void load32(uint32_t at, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(at));
}
__device__ __forceinline__ void loaded(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                   "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                   "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :: "memory");
}
__device__ __forceinline__ void store16(uint32_t at, const uint32_t* w) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :: "r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]),
                    "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
                 : "memory");
}
__device__ __forceinline__ void store32(uint32_t at, const float (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 :: "r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
                    "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
                    "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]),
                    "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31])
                 : "memory");
}
// The same for 64 columns of 16 rows, as a warp's product fragments lie: v[4 i + 2 r
// + c] is row 8 r + lane / 4, column 8 i + 2 (lane mod 4) + c
__device__ __forceinline__ void load_rows16(uint32_t at, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(at));
}
// and 32 words (64 bf16 columns) of 16 rows: w[2 i + r] is row 8 r + lane / 4, word
// 4 i + lane mod 4
__device__ __forceinline__ void store_rows16(uint32_t at, const uint32_t (&w)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :: "r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]),
                    "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
                 : "memory");
}
__device__ __forceinline__ void stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void alloc_all(uint32_t slot) {       // the whole tensor memory of the SM
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(slot) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void free_all(uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(at) : "memory");
}

// 64 channels of 128 rows of one head: coordinates channel, head, row
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int channel, int head, int row, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(channel), "r"(head), "r"(row), "r"(bar) : "memory");
}
// a tile of DP channels, announced on its barrier
template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int head, int row, uint32_t bar) {
    mbar_arrive_tx(bar, DP / BOX * BOX_BYTES);
#pragma unroll
    for (int b = 0; b < DP / BOX; ++b) load_box(dst + b * BOX_BYTES, map, b * BOX, head, row, bar);
}
// Rows from `from` on of a tile of DP channels become zero: rows behind a
// sequence's end, whose contents (another sequence's, or anything) must not meet a
// weight of 0 in a product.  By a whole warp, before the products read the tile.
template <int DP>
__device__ __forceinline__ void clear_rows(unsigned char* tile, int from) {
    if (from >= ROWS) return;
    const int lane = threadIdx.x & 31;
    for (int b = 0; b < DP / BOX; ++b)
        for (int i = from * 8 + lane; i < ROWS * 8; i += 32)
            reinterpret_cast<uint4*>(tile + b * BOX_BYTES)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    __syncwarp();
}

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool probe(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded waits of a CTA.  A wait that gives up sets the flag, and with it every
// other wait of the CTA ends.  With a limit of 0 only what has happened by the first
// probe counts.
static __device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, uint64_t limit_ns, volatile int* gave_up) {
    WaitClock clock;
    for (int spin = 0; limit_ns && spin < MBAR_SPIN_LIMIT; ++spin) {
        if (probe(bar, parity)) return true;
        if ((spin & 31) == 31 && ((gave_up && *gave_up) || clock.look(now_ns(), limit_ns))) break;
    }
    if (gave_up) *gave_up = 1;
    return false;
}
struct Waits {
    uint64_t limit_ns;
    volatile int* gave_up;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
        return probe(bar, parity) || wait_long(bar, parity, limit_ns, gave_up);
    }
    // one answer for the whole warp
    __device__ __forceinline__ bool warp(uint32_t bar, uint32_t parity) const {
        if (__all_sync(0xFFFFFFFFu, probe(bar, parity))) return true;
        return __all_sync(0xFFFFFFFFu, wait_long(bar, parity, limit_ns, gave_up));
    }
    // for what is in flight in any case (a copy, a product): not cut short by the flag
    __device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) const { wait_long(bar, parity, 2000000000u, nullptr); }
};

// two binary32 numbers at a time
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
__device__ __forceinline__ uint32_t bf16_of(uint64_t v) {
    float a, b;
    parts_of(v, a, b);
    return f32_to_bf16x2(a, b);
}
// the largest of three; a NaN counts as nothing
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void arrive_warp(uint32_t bar) {      // one arrival for the warp's accesses so far
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

__device__ __forceinline__ unsigned char* align1024(unsigned char* p) {
    return reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(p) + 1023) & ~(uintptr_t)1023);
}

// One row of an accumulator out, 32 columns at a time: all lanes call it.  Whether
// all it wrote is finite.
template <typename O, int DP>
__device__ __forceinline__ bool write_row(uint32_t at, O* row, bool valid, int dim, bool vec, float by, bool nan, bool none) {
    float odd = 0.0f;                  // 0, or NaN after a value that is not finite
#pragma unroll
    for (int c = 0; c < DP; c += 32) {
        float v[32];
        __syncwarp();                  // a load of tensor memory takes all lanes
        if (!none) {
            load32(at + c, v);
            loaded(v);
        }
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            if (!valid || c + j >= dim) continue;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = nan ? __int_as_float(0x7FFFFFFF) : none ? 0.0f : v[j + i] * by;
                odd = fmaf(x[i], 0.0f, odd);
            }
            if (vec) put8(row + c + j, x);
            else store8<false>(row, c + j, dim, x);
        }
    }
    return odd == 0.0f;
}

// Host: the tensor map of a matrix of heads, boxes of 64 channels x 1 head x 128
// rows in the 128-byte swizzle; channels past the head's and rows past the matrix
// read as zero.  Rows and heads must start on 16-byte boundaries.
int head_map(CUtensorMap* map, const void* base, long long rows, int heads, int head_dim, long long ld);

}  // namespace tc
}  // namespace iso
