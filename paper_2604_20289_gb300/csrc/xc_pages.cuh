// What the kernels that plan page operations share (k_kv_pages.cu, k_kv_evict.cu).
#pragma once
#include "xc_branch.cuh"

namespace xc {

constexpr int PLAN_THREADS = KV_LIST_MAX;   // a thread for every listed sequence

// Exclusive scan over the CTA; `total` receives the sum.  Every thread calls it.
__device__ __forceinline__ int block_scan(int v, int *sh, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                       // sh is free
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int s = sh[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += y;
        }
        sh[lane] = s;
    }
    __syncthreads();
    total = sh[31];
    return x - v + (warp > 0 ? sh[warp - 1] : 0);
}

// Writes the ids p in [lo, hi) with (ref[p] > 0) == used, ascending, to out
// until `most` are found; returns how many were written (CTA-uniform).
static __device__ int list_pages(const int *ref, int lo, int hi, bool used, int most, int *out, int *sh) {
    constexpr int PER = 8;
    int have = 0;
    for (int base = lo; base < hi && have < most; base += PLAN_THREADS * PER) {
        const int p0 = base + (int)threadIdx.x * PER;
        unsigned hit = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (p0 + i < hi && (ref[p0 + i] > 0) == used) hit |= 1u << i;
        int total;
        int at = have + block_scan(__popc(hit), sh, total);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (hit >> i & 1u) {
                if (at < most) out[at] = p0 + i;
                ++at;
            }
        have += total;
    }
    __syncthreads();
    return have < most ? have : most;
}

struct KvState {
    int n_pages, ps, max_seqs, max_pages;
    int *ref, *table, *len;
};
static KvState kv_state(const xc_kv_cache &c) {
    return KvState{c.n_pages, c.page_size, c.max_seqs, c.max_pages, c.ref, c.table, c.len};
}

}  // namespace xc
