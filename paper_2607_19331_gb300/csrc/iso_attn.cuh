// iso_attn.cuh -- what the attention kernels share: arguments, the sequences'
// tiles and what a query sees.
#pragma once

#include "iso_train.cuh"
#include "iso_internal.cuh"

#include <atomic>

namespace iso {

// Dynamic shared memory beyond the default for a kernel, asked for once a device
// (`done` belongs to the kernel)
template <typename K>
int allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return ISO_ERR_CUDA;
    const uint64_t bit = dev < 64 ? 1ULL << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return ISO_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return ISO_ERR_CUDA;
    done.fetch_or(bit, std::memory_order_relaxed);
    return ISO_OK;
}

struct AttnArgs {
    const void *q, *k, *v;
    long long ldq, ldk, ldv;
    const void* out;             // forward: written; backward: read
    long long ldo;
    float* lse;                  // [heads][q_rows]
    int32_t q_rows, k_rows;
    int32_t heads, group, head_dim;     // group: query heads of a key head
    int32_t causal;
    long long window;            // 0: none
    float scale;
    int32_t n_seqs;              // 0: one sequence of all rows
    const int32_t *q_ends, *k_ends;
    int32_t* status;
    // backward
    const void* dout;
    long long lddo;
    void *dq, *dk, *dv;
    long long lddq, lddk, lddv;
    float* delta;                // [heads][q_rows]
};

// A tile of one sequence: its rows are first .. first + BM - 1 of the sequence's.
struct AttnTile {
    int q0, nq, k0, nk;          // the sequence: first query, queries, first key, keys
    int first;
};

// Tiles that hold every sequence whatever the offsets say (host).
inline long long attn_tiles(long long rows, long long n_seqs, int bm) {
    return rows / bm + (n_seqs ? n_seqs : 1);
}

__device__ __forceinline__ void attn_span(const int32_t* ends, int i, int rows, int& at, int& n, bool& bad) {
    const int a = ends[i], b = ends[i + 1];
    bad |= a < 0 || b < a || b > rows;
    at = min(max(a, 0), rows);
    n = min(max(b, at), rows) - at;
}

// Tile `index` over the sequences' queries (over_keys: their keys), bm rows each;
// false where there are fewer.  Called by whole warps; every lane gets the same.
// A sequence's last tile comes first: with causal it has the most keys.
__device__ __forceinline__ bool attn_find_tile(const AttnArgs& g, int index, int bm, bool over_keys, AttnTile& t) {
    if (g.n_seqs == 0) {
        t = {0, g.q_rows, 0, g.k_rows, 0};
        const int n = over_keys ? g.k_rows : g.q_rows, tiles = (n + bm - 1) / bm;
        if (index >= tiles) return false;
        t.first = (over_keys ? index : tiles - 1 - index) * bm;     // the tiles with the most work first
        return true;
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int s = 0; s < g.n_seqs; s += 32) {
        int q0 = 0, nq = 0, k0 = 0, nk = 0;
        bool bad = false;
        if (s + lane < g.n_seqs) {
            attn_span(g.q_ends, s + lane, g.q_rows, q0, nq, bad);
            attn_span(g.k_ends, s + lane, g.k_rows, k0, nk, bad);
        }
        if (bad && g.status) atomicCAS(g.status, 0, (int32_t)ISO_ERR_INDEX);
        const int n = over_keys ? nk : nq, tiles = (int)(((long long)n + bm - 1) / bm);
        int sum = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += x;
        }
        const unsigned hit = __ballot_sync(0xFFFFFFFFu, before + sum > index);
        if (hit) {
            const int l = __ffs(hit) - 1;
            const int in = index - (before + __shfl_sync(0xFFFFFFFFu, sum - tiles, l)), of = __shfl_sync(0xFFFFFFFFu, tiles, l);
            t.q0 = __shfl_sync(0xFFFFFFFFu, q0, l);
            t.nq = __shfl_sync(0xFFFFFFFFu, nq, l);
            t.k0 = __shfl_sync(0xFFFFFFFFu, k0, l);
            t.nk = __shfl_sync(0xFFFFFFFFu, nk, l);
            t.first = (over_keys ? in : of - 1 - in) * bm;
            return true;
        }
        before += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    return false;
}

// The keys that query i of the sequence sees: [lo, hi).
__device__ __forceinline__ void attn_keys_of(const AttnArgs& g, const AttnTile& t, int i, int& lo, int& hi) {
    lo = 0;
    hi = t.nk;
    if (g.causal) {
        const long long at = (long long)i + t.nk - t.nq;
        hi = (int)max(0LL, min((long long)t.nk, at + 1));
        if (g.window) lo = (int)max(0LL, min((long long)t.nk, at - g.window + 1));
    }
}
// The queries that see key j: [lo, hi).
__device__ __forceinline__ void attn_queries_of(const AttnArgs& g, const AttnTile& t, int j, int& lo, int& hi) {
    lo = 0;
    hi = t.nq;
    if (g.causal) {
        const long long at = (long long)j - (t.nk - t.nq);
        lo = (int)max(0LL, min((long long)t.nq, at));
        if (g.window) hi = (int)max(0LL, min((long long)t.nq, at + g.window));
    }
}

}  // namespace iso
