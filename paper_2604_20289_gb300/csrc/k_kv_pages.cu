// Pages of the branched key / value cache: fork, extend, free, compact, and
// the head-wise norm + rotation that fills it.
//
// The page state (reference counts, tables, lengths) is small and integer; one
// CTA plans a call over it, in the order the interface promises, and a second
// kernel over the whole GPU moves the pages it listed.  A plan validates its
// whole input before it writes anything.
#include "xc_branch.cuh"

namespace xc {

// Workspace (ints): copy list (source page, destination page, rows) with its
// length, free page ids, marks per sequence, new id per page.
struct KvPlan {
    int *n_copy, *n_live;
    int *src, *dst, *rows;      // [cap]
    int *free_ids;              // [n_pages]
    int *mark;                  // [max_seqs]
    int *map;                   // [n_pages]
};
static size_t kv_cap(const xc_kv_cache &c) { return c.n_pages > c.max_seqs ? c.n_pages : c.max_seqs; }
size_t kv_workspace_bytes(const xc_kv_cache &c) {
    return (4 + 3 * kv_cap(c) + 2 * (size_t)c.n_pages + c.max_seqs) * sizeof(int);
}
static KvPlan kv_plan(const xc_kv_cache &c, void *ws) {
    const size_t cap = kv_cap(c);
    int *p = reinterpret_cast<int *>(ws);
    KvPlan k;
    k.n_copy = p;
    k.n_live = p + 1;
    k.src = p + 4;
    k.dst = k.src + cap;
    k.rows = k.dst + cap;
    k.free_ids = k.rows + cap;
    k.mark = k.free_ids + c.n_pages;
    k.map = k.mark + c.max_seqs;
    return k;
}

constexpr int PLAN_THREADS = 1024;

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
__device__ int list_pages(const int *ref, int lo, int hi, bool used, int most, int *out, int *sh) {
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

__global__ void __launch_bounds__(PLAN_THREADS)
    kv_fork_plan_kernel(const KvState c, const int n, const int *src, const int *dst, const KvPlan pl, int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32], bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        bad = 0;
        *pl.n_copy = 0;
    }
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS) {
        const int s = src[i], d = dst[i];
        if (s < 0 || s >= c.max_seqs || d < 0 || d >= c.max_seqs) {
            bad = 1;
        } else {
            pl.mark[s] = 0;
            pl.mark[d] = 0;
        }
    }
    __syncthreads();
    if (!bad)
        for (int i = tid; i < n; i += PLAN_THREADS) {
            const int l = c.len[src[i]];
            if (atomicAdd(&pl.mark[dst[i]], 1) > 0 || c.len[dst[i]] != 0 || l < 0 ||
                (long long)l > (long long)c.max_pages * c.ps)
                bad = 1;
        }
    __syncthreads();
    if (!bad)
        for (int i = warp; i < n; i += PLAN_THREADS / 32) {   // no source is a destination; its pages exist
            const int s = src[i], np = (c.len[s] + c.ps - 1) / c.ps;
            if (pl.mark[s] != 0) bad = 1;
            for (int j = lane; j < np; j += 32) {
                const int p = c.table[(size_t)s * c.max_pages + j];
                if (p < 0 || p >= c.n_pages) bad = 1;
            }
        }
    __syncthreads();
    if (bad) {
        if (tid == 0 && err) atomicOr(err, ERR_BAD_SEQ);
        return;
    }
    int need = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        int total;
        block_scan(i < n && c.len[src[i]] % c.ps != 0 ? 1 : 0, sh, total);
        need += total;
    }
    if (list_pages(c.ref, 0, c.n_pages, false, need, pl.free_ids, sh) < need) {
        if (tid == 0 && err) atomicOr(err, ERR_CACHE_FULL);
        return;
    }
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        const int l = i < n ? c.len[src[i]] : 0;
        const int part = l % c.ps, full = l / c.ps;
        int total;
        const int at = base + block_scan(part != 0 ? 1 : 0, sh, total);
        if (part != 0) {
            const int fresh = pl.free_ids[at];
            c.ref[fresh] = 1;
            c.table[(size_t)dst[i] * c.max_pages + full] = fresh;
            pl.src[at] = c.table[(size_t)src[i] * c.max_pages + full];
            pl.dst[at] = fresh;
            pl.rows[at] = part;
        }
        if (i < n) c.len[dst[i]] = l;
        base += total;
    }
    if (tid == 0) *pl.n_copy = need;
    for (int i = warp; i < n; i += PLAN_THREADS / 32) {
        const int s = src[i], d = dst[i], full = c.len[s] / c.ps;
        for (int j = lane; j < full; j += 32) {
            const int p = c.table[(size_t)s * c.max_pages + j];
            c.table[(size_t)d * c.max_pages + j] = p;
            atomicAdd(&c.ref[p], 1);
        }
    }
}

__global__ void __launch_bounds__(PLAN_THREADS)
    kv_extend_kernel(const KvState c, const int n, const int *seqs, const int n_new, int *slots, const KvPlan pl,
                     int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32], bad;
    __shared__ unsigned long long want;
    const int tid = threadIdx.x;
    const long long n_slots = (long long)n * n_new;
    if (tid == 0) {
        bad = 0;
        want = 0;
    }
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS) {
        const int s = seqs[i];
        if (s < 0 || s >= c.max_seqs) bad = ERR_BAD_SEQ;
        else pl.mark[s] = 0;
    }
    __syncthreads();
    if (!bad)
        for (int i = tid; i < n; i += PLAN_THREADS) {
            const int s = seqs[i], l = c.len[s];
            if (atomicAdd(&pl.mark[s], 1) > 0 || l < 0) {
                atomicOr(&bad, ERR_BAD_SEQ);
            } else if ((long long)l + n_new > (long long)c.max_pages * c.ps) {
                atomicOr(&bad, ERR_CACHE_FULL);
            } else if (l % c.ps != 0) {          // the last page is written: it must be this sequence's own
                const int p = c.table[(size_t)s * c.max_pages + l / c.ps];
                if (p < 0 || p >= c.n_pages || c.ref[p] != 1) atomicOr(&bad, ERR_BAD_SEQ);
            }
        }
    __syncthreads();
    int need = 0;
    if (!bad) {
        for (int i = tid; i < n; i += PLAN_THREADS) {
            const int l = c.len[seqs[i]];
            atomicAdd(&want, (unsigned long long)((l + n_new + c.ps - 1) / c.ps - (l + c.ps - 1) / c.ps));
        }
        __syncthreads();
        if (want <= (unsigned long long)c.n_pages) need = (int)want;
        else if (tid == 0) bad = ERR_CACHE_FULL;
        __syncthreads();
    }
    if (!bad && list_pages(c.ref, 0, c.n_pages, false, need, pl.free_ids, sh) < need) {
        __syncthreads();
        if (tid == 0) bad = ERR_CACHE_FULL;
    }
    __syncthreads();
    if (bad) {
        for (long long e = tid; e < n_slots; e += PLAN_THREADS) slots[e] = -1;
        if (tid == 0 && err) atomicOr(err, bad);
        return;
    }
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        const int s = i < n ? seqs[i] : 0, l = i < n ? c.len[s] : 0;
        const int have = (l + c.ps - 1) / c.ps;
        const int k = i < n ? (l + n_new + c.ps - 1) / c.ps - have : 0;
        int total;
        const int at = base + block_scan(k, sh, total);
        for (int j = 0; j < k; ++j) {
            const int p = pl.free_ids[at + j];
            c.ref[p] = 1;
            c.table[(size_t)s * c.max_pages + have + j] = p;
        }
        if (i < n) c.len[s] = l + n_new;
        base += total;
    }
    __syncthreads();
    for (long long e = tid; e < n_slots; e += PLAN_THREADS) {
        const int i = (int)(e / n_new), s = seqs[i];
        const int at = c.len[s] - n_new + (int)(e - (long long)i * n_new);
        slots[e] = c.table[(size_t)s * c.max_pages + at / c.ps] * c.ps + at % c.ps;
    }
}

// One CTA per listed sequence.  The exchange of len makes a sequence that is
// listed twice release its pages once.
__global__ void __launch_bounds__(256) kv_free_kernel(const KvState c, const int *seqs, int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int l_sh;
    const int s = seqs[blockIdx.x];
    if (s < 0 || s >= c.max_seqs) {
        if (threadIdx.x == 0 && err) atomicOr(err, ERR_BAD_SEQ);
        return;
    }
    if (threadIdx.x == 0) l_sh = atomicExch(&c.len[s], 0);
    __syncthreads();
    const long long np = ((long long)l_sh + c.ps - 1) / c.ps;
    if (l_sh < 0 || np > c.max_pages) {
        if (threadIdx.x == 0 && err) atomicOr(err, ERR_BAD_SEQ);
        return;
    }
    for (int j = threadIdx.x; j < (int)np; j += blockDim.x) {
        const int p = c.table[(size_t)s * c.max_pages + j];
        c.table[(size_t)s * c.max_pages + j] = -1;
        if (p < 0 || p >= c.n_pages) {
            if (err) atomicOr(err, ERR_BAD_SEQ);
        } else {
            atomicSub(&c.ref[p], 1);
        }
    }
}

__global__ void __launch_bounds__(PLAN_THREADS) kv_compact_plan_kernel(const KvState c, const KvPlan pl, int *n_live) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32];
    const int tid = threadIdx.x;
    int mine = 0, live;
    for (int p = tid; p < c.n_pages; p += PLAN_THREADS) mine += c.ref[p] > 0 ? 1 : 0;
    block_scan(mine, sh, live);
    const int n = list_pages(c.ref, 0, live, false, live, pl.dst, sh);          // holes
    list_pages(c.ref, live, c.n_pages, true, n, pl.src, sh);                     // as many pages past the end
    for (int p = live + tid; p < c.n_pages; p += PLAN_THREADS) pl.map[p] = p;
    __syncthreads();
    for (int k = tid; k < n; k += PLAN_THREADS) {
        const int a = pl.src[k], b = pl.dst[k];
        pl.rows[k] = c.ps;
        pl.map[a] = b;
        c.ref[b] = c.ref[a];
        c.ref[a] = 0;
    }
    if (tid == 0) {
        *pl.n_copy = n;
        *pl.n_live = live;
        *n_live = live;
    }
}

// Copies the listed pages' rows in every layer of both pools: 16 KB chunks,
// four 16-byte loads in flight per thread.  With n_entries > 0 also renames
// the table entries of moved pages.  HBM bound: twice the bytes of the rows.
constexpr int COPY_VECS = 1024;
__global__ void __launch_bounds__(256)
    kv_copy_kernel(uint4 *k, uint4 *v, const int n_layers, const int n_pages, const int ps, const int row_vecs,
                   const KvPlan pl, int *table, const long long n_entries) {
    pdl_wait();
    if (n_entries > 0) {
        const int live = *pl.n_live;
        for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < n_entries; e += (long long)gridDim.x * 256) {
            const int p = table[e];
            if (p >= live && p < n_pages) table[e] = pl.map[p];
        }
    }
    const int n = *pl.n_copy;
    const int page_vecs = ps * row_vecs;
    const int per = (page_vecs + COPY_VECS - 1) / COPY_VECS;
    const long long total = (long long)n * n_layers * 2 * per;
    for (long long w = blockIdx.x; w < total; w += gridDim.x) {
        const long long item = w / per;
        const int off = (int)(w - item * per) * COPY_VECS + threadIdx.x;
        const int i = (int)(item % n), lk = (int)(item / n);
        const int vecs = pl.rows[i] * row_vecs;
        uint4 *pool = (lk & 1) ? v : k;
        const size_t layer = (size_t)(lk >> 1) * n_pages;
        const uint4 *src = pool + (layer + pl.src[i]) * page_vecs;
        uint4 *dst = pool + (layer + pl.dst[i]) * page_vecs;
        uint4 t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (off + 256 * j < vecs) t[j] = __ldcs(src + off + 256 * j);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (off + 256 * j < vecs) __stcs(dst + off + 256 * j, t[j]);
    }
}

static cudaError_t launch_copy(const xc_kv_cache &c, const KvPlan &pl, long long n_entries, cudaStream_t st) {
    return launch_pdl(kv_copy_kernel, dim3(device_sms() * 8), dim3(256), 0, st, reinterpret_cast<uint4 *>(c.k),
                      reinterpret_cast<uint4 *>(c.v), c.n_layers, c.n_pages, c.page_size,
                      (int)(kv_row_bytes(c) / 16), pl, c.table, n_entries);
}

cudaError_t kv_fork(const xc_kv_cache &c, int n, const int *src, const int *dst, void *ws, int *err, cudaStream_t st) {
    const KvPlan pl = kv_plan(c, ws);
    cudaError_t e = launch_pdl(kv_fork_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, kv_state(c), n, src, dst, pl, err);
    if (e != cudaSuccess) return e;
    return launch_copy(c, pl, 0, st);
}
cudaError_t kv_extend(const xc_kv_cache &c, int n, const int *seqs, int n_new, int *slots, void *ws, int *err,
                      cudaStream_t st) {
    return launch_pdl(kv_extend_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, kv_state(c), n, seqs, n_new, slots,
                      kv_plan(c, ws), err);
}
cudaError_t kv_free(const xc_kv_cache &c, int n, const int *seqs, int *err, cudaStream_t st) {
    return launch_pdl(kv_free_kernel, dim3(n), dim3(256), 0, st, kv_state(c), seqs, err);
}
cudaError_t kv_compact(const xc_kv_cache &c, int *n_live, void *ws, cudaStream_t st) {
    const KvPlan pl = kv_plan(c, ws);
    cudaError_t e = launch_pdl(kv_compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, kv_state(c), pl, n_live);
    if (e != cudaSuccess) return e;
    return launch_copy(c, pl, (long long)c.max_seqs * c.max_pages, st);
}

// ------------------------------------------------------- rotation and norm
__global__ void rope_axes_table_kernel(const RopeAxes ax, const double theta, float2 *out, const long long n) {
    pdl_wait();
    pdl_release();
    long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (e >= n) return;
    float2 *dst = out + e;
    int a = 0;
    for (; a + 1 < ax.n; ++a) {
        const long long span = (long long)ax.n_pos[a] * ax.pairs[a];
        if (e < span) break;
        e -= span;
    }
    const int pairs = ax.pairs[a];
    const int p = (int)(e / pairs), j = (int)(e % pairs);
    double s, c;
    sincos((double)p * pow(theta, -(double)j / pairs), &s, &c);
    *dst = make_float2((float)c, (float)s);
}
cudaError_t rope_axes_table(const RopeAxes &ax, double theta, float2 *out, cudaStream_t st) {
    long long n = 0;
    for (int a = 0; a < ax.n; ++a) n += (long long)ax.pairs[a] * ax.n_pos[a];
    return launch_pdl(rope_axes_table_kernel, dim3((unsigned)((n + 127) / 128)), dim3(128), 0, st, ax, theta, out, n);
}

// 16 bytes of a row as floats, and back (rounded once).
template <typename T> __device__ __forceinline__ void unpack(const uint4 &u, float (&x)[16 / sizeof(T)]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}
template <typename T> __device__ __forceinline__ uint4 pack(const float (&x)[16 / sizeof(T)]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            w[j] = __float_as_uint(x[j]);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// y = rot(x / sqrt(mean x^2 + eps) * gamma) per head; q -> q_out, k and v ->
// the token's cache row.  A warp takes one token and SEG passes over its
// query, its key or its value heads; a lane holds 16 bytes of a head, LPH =
// head bytes / 16 lanes a head (the sum of squares and the halves' partners
// by shuffles).  Gain and rotation are folded once per warp,
//   y_a = r (x_a (g_a c) - x_b (g_b s)),  y_b = r (x_a (g_a s) + x_b (g_b c)),
// r the reciprocal root, so a lane's factors stay in registers over the
// passes.  HBM bound, every input and output byte once; the SEG input loads
// are issued before anything waits for the token's position and slot.
template <typename T, int HD, bool HALF, int SEG>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const NormRopeArgs a, const int seg_q, const int seg_k) {
    pdl_wait();
    pdl_release();
    constexpr int VPT = 16 / sizeof(T), LPH = HD / VPT, HPW = 32 / LPH;
    const int lane = threadIdx.x & 31, li = lane % LPH;
    const int n_seg = seg_q + 2 * seg_k, item = blockIdx.x * 8 + (threadIdx.x >> 5), t = item / n_seg;
    if (t >= a.T) return;
    int seg = item - t * n_seg;
    const int kind = seg < seg_q ? 0 : seg < seg_q + seg_k ? 1 : 2;       // queries, keys, values
    seg -= kind == 0 ? 0 : kind == 1 ? seg_q : seg_q + seg_k;
    const int heads = kind == 0 ? a.H : a.Hk, hw = seg * (SEG * HPW), h0 = hw + lane / LPH;
    const T *src = (kind == 0   ? reinterpret_cast<const T *>(a.q) + (size_t)t * a.q_ld
                    : kind == 1 ? reinterpret_cast<const T *>(a.k) + (size_t)t * a.k_ld
                                : reinterpret_cast<const T *>(a.v) + (size_t)t * a.v_ld) + h0 * HD + li * VPT;
    uint4 in[SEG];
#pragma unroll
    for (int u = 0; u < SEG; ++u) {
        in[u] = make_uint4(0, 0, 0, 0);
        if (h0 + u * HPW < heads) in[u] = *reinterpret_cast<const uint4 *>(src + u * (HPW * HD));
    }
    const long slot = a.slots[t];
    bool ok = slot >= -1 && slot < a.n_rows;
    int base[ROPE_AXES];                                   // table entry of (position, pair 0) of each axis
    int at = 0, first = 0;
#pragma unroll
    for (int x = 0; x < ROPE_AXES; ++x) {
        base[x] = 0;
        if (x < a.ax.n) {
            const int pos = a.pos[(size_t)t * a.ax.n + x];
            if (pos < 0 || pos >= a.ax.n_pos[x]) ok = false;
            base[x] = at + pos * a.ax.pairs[x] - first;
            at += a.ax.n_pos[x] * a.ax.pairs[x];
            first += a.ax.pairs[x];
        }
    }
    if (!ok) {
        if (lane == 0 && item == t * n_seg && a.err) atomicOr(a.err, ERR_BAD_POS);
        return;
    }
    if (kind != 0 && slot < 0) return;                     // a token that keeps no keys
    T *dst = (kind == 0 ? reinterpret_cast<T *>(a.q_out) + (size_t)t * a.o_ld
                        : reinterpret_cast<T *>(kind == 1 ? a.k_pool : a.v_pool) + (size_t)slot * a.Hk * HD) + h0 * HD + li * VPT;
    if (kind == 2) {
#pragma unroll
        for (int u = 0; u < SEG; ++u)
            if (h0 + u * HPW < heads) *reinterpret_cast<uint4 *>(dst + u * (HPW * HD)) = in[u];
        return;
    }
    // factors of the lane's element j and of its partner
    const float *gamma = kind == 0 ? a.gamma_q : a.gamma_k;
    const int mate = HALF ? (li * VPT + HD / 2) % HD : li * VPT;
    float g[VPT], gm[VPT], fx[VPT], fo[VPT];
#pragma unroll
    for (int j = 0; j < VPT; j += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(gamma + li * VPT + j), y = *reinterpret_cast<const float4 *>(gamma + mate + j);
        g[j] = x.x; g[j + 1] = x.y; g[j + 2] = x.z; g[j + 3] = x.w;
        gm[j] = y.x; gm[j + 1] = y.y; gm[j + 2] = y.z; gm[j + 3] = y.w;
    }
#pragma unroll
    for (int j = 0; j < VPT; j += HALF ? 1 : 2) {
        const int p = HALF ? (li * VPT + j) % (HD / 2) : (li * VPT + j) / 2;
        int b = base[0], end = a.ax.pairs[0];
#pragma unroll
        for (int x = 1; x < ROPE_AXES; ++x)
            if (x < a.ax.n && p >= end) {
                b = base[x];
                end += a.ax.pairs[x];
            }
        const float2 cs = a.table[b + p];
        if constexpr (HALF) {
            fx[j] = g[j] * cs.x;
            fo[j] = gm[j] * (li < LPH / 2 ? -cs.y : cs.y);
        } else {
            fx[j] = g[j] * cs.x;
            fo[j] = -g[j + 1] * cs.y;
            fx[j + 1] = g[j + 1] * cs.x;
            fo[j + 1] = g[j] * cs.y;
        }
    }
#pragma unroll
    for (int u = 0; u < SEG; ++u) {
        if (hw + u * HPW >= heads) break;                  // the whole warp is past the last head
        float x[VPT], o[VPT], y[VPT];
        unpack<T>(in[u], x);
        float ss = 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) ss = fmaf(x[j], x[j], ss);
#pragma unroll
        for (int d = LPH / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float r = rsqrtf(ss * (1.0f / HD) + a.eps);
        if constexpr (HALF) {
            uint4 other;
            other.x = __shfl_xor_sync(0xffffffffu, in[u].x, LPH / 2);
            other.y = __shfl_xor_sync(0xffffffffu, in[u].y, LPH / 2);
            other.z = __shfl_xor_sync(0xffffffffu, in[u].z, LPH / 2);
            other.w = __shfl_xor_sync(0xffffffffu, in[u].w, LPH / 2);
            unpack<T>(other, o);
        } else {
#pragma unroll
            for (int j = 0; j < VPT; ++j) o[j] = x[j ^ 1];
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) y[j] = r * fmaf(o[j], fo[j], x[j] * fx[j]);
        if (h0 + u * HPW < heads) *reinterpret_cast<uint4 *>(dst + u * (HPW * HD)) = pack<T>(y);
    }
}

template <typename T, int HD, int SEG>
static cudaError_t launch_norm_rope(bool half, const NormRopeArgs &a, cudaStream_t st) {
    constexpr int PER = SEG * (32 / (HD * (int)sizeof(T) / 16));          // heads of a warp
    const int seg_q = (a.H + PER - 1) / PER, seg_k = (a.Hk + PER - 1) / PER;
    const dim3 grid((unsigned)(((long long)a.T * (seg_q + 2 * seg_k) + 7) / 8));
    return half ? launch_pdl(qk_norm_rope_kernel<T, HD, true, SEG>, grid, dim3(256), 0, st, a, seg_q, seg_k)
                : launch_pdl(qk_norm_rope_kernel<T, HD, false, SEG>, grid, dim3(256), 0, st, a, seg_q, seg_k);
}
// Passes a warp: 4 where that many still fill the SMs with 16 warps each (12960
// tokens of 3 x 40 heads x 128, bf16, 796 MB: 116 us at 4 passes, 6.9 TB/s;
// 131 at 8, 145 at 2, 237 at 1; 4099 tokens of 40 + 2 x 8 heads x 64: 15.8 /
// 19.1 / 16.5 / 26.9 us), one for few tokens, whose latency is the passes'
// (8 tokens of 3 x 40 heads x 128: 2.5 us).
template <typename T, int HD>
static cudaError_t launch_norm_rope(bool half, const NormRopeArgs &a, cudaStream_t st) {
    const long long passes = (long long)a.T * ((a.H + 2ll * a.Hk) * HD * (int)sizeof(T) / 512 + 1);
    return passes / 4 >= 16ll * device_sms() ? launch_norm_rope<T, HD, 4>(half, a, st) : launch_norm_rope<T, HD, 1>(half, a, st);
}
template <typename T> static cudaError_t norm_rope_hd(int hd, bool half, const NormRopeArgs &a, cudaStream_t st) {
    switch (hd) {
        case 16: return launch_norm_rope<T, 16>(half, a, st);
        case 32: return launch_norm_rope<T, 32>(half, a, st);
        case 64: return launch_norm_rope<T, 64>(half, a, st);
        case 128: return launch_norm_rope<T, 128>(half, a, st);
    }
    return cudaErrorInvalidValue;
}
cudaError_t qk_norm_rope(int dtype, int head_dim, bool half_split, const NormRopeArgs &a, cudaStream_t st) {
    return dtype == XC_BF16 ? norm_rope_hd<bf16>(head_dim, half_split, a, st)
                            : norm_rope_hd<float>(head_dim, half_split, a, st);
}

}  // namespace xc
