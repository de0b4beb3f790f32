// Pages of the branched key / value cache: fork, extend, free, compact, and
// the head-wise norm + rotation that fills it.
//
// The page state (reference counts, tables, lengths) is small and integer; one
// CTA plans a call over it, in the order the interface promises, and a second
// kernel over the whole GPU moves the pages it listed.  A plan validates its
// whole input before it writes anything.
#include <algorithm>

#include "xc_branch.cuh"
#include "xc_pages.cuh"

namespace xc {

// Workspace (ints): copy list (source page, destination page, rows) with its
// length, free page ids, new id per page.
struct KvPlan {
    int *n_copy, *n_live;
    int *src, *dst, *rows;      // [n_pages]
    int *free_ids;              // [n_pages]
    int *map;                   // [n_pages]
};
size_t kv_workspace_bytes(const xc_kv_cache &c) { return (4 + 5 * (size_t)c.n_pages) * sizeof(int); }
static KvPlan kv_plan(const xc_kv_cache &c, void *ws) {
    int *p = reinterpret_cast<int *>(ws);
    KvPlan k;
    k.n_copy = p;
    k.n_live = p + 1;
    k.src = p + 4;
    k.dst = k.src + c.n_pages;
    k.rows = k.dst + c.n_pages;
    k.free_ids = k.rows + c.n_pages;
    k.map = k.free_ids + c.n_pages;
    return k;
}

// Latency bound (one CTA, a few dependent loads), so each thread keeps its pair
// in registers and the free pages are listed while the lengths are on their
// way: 6 us for 4 pairs and 7 for 16, where a version that re-read them per step
// took 10 and 11.
__global__ void __launch_bounds__(PLAN_THREADS)
    kv_fork_plan_kernel(const KvState c, const int n, const int *src, const int *dst, const KvPlan pl, int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32], sh_src[PLAN_THREADS], sh_dst[PLAN_THREADS], sh_pages[PLAN_THREADS],
        sh_times[PLAN_THREADS];
    const int tid = threadIdx.x;
    const bool mine = tid < n;
    const int s = mine ? src[tid] : 0, d = mine ? dst[tid] : 0;
    bool bad = s < 0 || s >= c.max_seqs || d < 0 || d >= c.max_seqs;
    const int l = mine && !bad ? c.len[s] : 0, ld = mine && !bad ? c.len[d] : 0;
    sh_src[tid] = s;
    sh_dst[tid] = d;
    const int found = list_pages(c.ref, 0, c.n_pages, false, n, pl.free_ids, sh);
    if (tid == 0) *pl.n_copy = 0;
    bad = bad || ld != 0 || l < 0 || (long long)l > (long long)c.max_pages * c.ps;
    int times = 0;                                     // pairs that share this pair's source, at its first one
    if (mine)
        for (int j = 0; j < n; ++j) {                  // a destination listed twice, or a source that is one
            if ((j < tid && sh_dst[j] == d) || sh_dst[j] == s) bad = true;
            if (sh_src[j] == s) times = j < tid ? -n : times + 1;
        }
    sh_times[tid] = max(times, 0);
    sh_pages[tid] = mine && !bad ? (l + c.ps - 1) / c.ps : 0;
    const int full = l / c.ps, part = l - full * c.ps;
    bool any = __syncthreads_or(mine && bad);
    int last = -1;                                     // the page that is copied
    // 2^lg threads walk a pair's table row; the first KEEP ids of each stay in registers
    constexpr int KEEP = 8;
    const int lg = 31 - __clz(PLAN_THREADS / n), pair = tid >> lg, per = 1 << lg, j0 = tid & (per - 1);
    const int *row = c.table + (size_t)(pair < n ? sh_src[pair] : 0) * c.max_pages;
    int ids[KEEP];
    if (!any) {
        const int np = pair < n ? sh_pages[pair] : 0;
        bool wrong = false;
        if (mine && part != 0) last = c.table[(size_t)s * c.max_pages + full];
#pragma unroll
        for (int i = 0; i < KEEP; ++i) ids[i] = j0 + i * per < np ? row[j0 + i * per] : 0;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) wrong = wrong || ids[i] < 0 || ids[i] >= c.n_pages;
        for (int j = j0 + KEEP * per; j < np; j += per) wrong = wrong || row[j] < 0 || row[j] >= c.n_pages;
        any = __syncthreads_or(wrong);
    }
    if (any) {
        if (tid == 0 && err) atomicOr(err, ERR_BAD_SEQ);
        return;
    }
    int need;
    const int at = block_scan(mine && part != 0 ? 1 : 0, sh, need);
    if (found < need) {
        if (tid == 0 && err) atomicOr(err, ERR_CACHE_FULL);
        return;
    }
    if (mine) {
        if (part != 0) {
            const int fresh = pl.free_ids[at];
            c.ref[fresh] = 1;
            c.table[(size_t)d * c.max_pages + full] = fresh;
            pl.src[at] = last;
            pl.dst[at] = fresh;
            pl.rows[at] = part;
        }
        c.len[d] = l;
    }
    if (tid == 0) *pl.n_copy = need;
    sh_pages[tid] = mine ? full : 0;
    __syncthreads();
    if (pair >= n) return;
    int *to = c.table + (size_t)sh_dst[pair] * c.max_pages;
    const int nf = sh_pages[pair], add = sh_times[pair];   // a page's count goes up once for all children of a source
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int j = j0 + i * per;
        if (j < nf) {
            to[j] = ids[i];
            if (add > 0) atomicAdd(&c.ref[ids[i]], add);
        }
    }
    for (int j = j0 + KEEP * per; j < nf; j += per) {
        const int p = row[j];
        to[j] = p;
        if (add > 0) atomicAdd(&c.ref[p], add);
    }
}

__global__ void __launch_bounds__(PLAN_THREADS)
    kv_extend_kernel(const KvState c, const int n, const int *seqs, const int n_new, int *slots, const KvPlan pl,
                     int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32], sh_seq[PLAN_THREADS], sh_len[PLAN_THREADS], sh_at[PLAN_THREADS], sh_k[PLAN_THREADS], why;
    __shared__ unsigned long long want;
    const int tid = threadIdx.x;
    const long long n_slots = (long long)n * n_new;
    const bool mine = tid < n;
    const int s = mine ? seqs[tid] : 0;
    int bad = s < 0 || s >= c.max_seqs ? ERR_BAD_SEQ : 0;
    const int l = mine && !bad ? c.len[s] : 0;
    sh_seq[tid] = s;
    if (tid == 0) {
        why = 0;
        want = 0;
    }
    const long long most = (long long)n * ((n_new + c.ps - 1) / c.ps);    // pages that n_new tokens may need
    const int found = list_pages(c.ref, 0, c.n_pages, false, (int)min(most, (long long)c.n_pages), pl.free_ids, sh);
    if (mine && !bad) {
        for (int j = 0; j < tid; ++j)
            if (sh_seq[j] == s) bad = ERR_BAD_SEQ;
        if (l < 0) bad = ERR_BAD_SEQ;
        else if ((long long)l + n_new > (long long)c.max_pages * c.ps) bad |= ERR_CACHE_FULL;
        if (!bad && l % c.ps != 0) {                   // the last page is written: it must be this sequence's own
            const int p = c.table[(size_t)s * c.max_pages + l / c.ps];
            if (p < 0 || p >= c.n_pages || c.ref[p] != 1) bad = ERR_BAD_SEQ;
        }
    }
    const int have = (l + c.ps - 1) / c.ps, k = mine && !bad ? (l + n_new + c.ps - 1) / c.ps - have : 0;
    if (mine && bad) atomicOr(&why, bad);
    if (k > 0) atomicAdd(&want, (unsigned long long)k);
    __syncthreads();
    const int fault = why != 0 ? why : want > (unsigned long long)found ? ERR_CACHE_FULL : 0;
    if (fault != 0) {
        for (long long e = tid; e < n_slots; e += PLAN_THREADS) slots[e] = -1;
        if (tid == 0 && err) atomicOr(err, fault);
        return;
    }
    int total;
    sh_at[tid] = block_scan(k, sh, total);
    sh_k[tid] = k;
    sh_len[tid] = l;
    if (mine) c.len[s] = l + n_new;
    __syncthreads();
    // 2^lg threads a sequence: its new pages, then its slots
    const int lg = 31 - __clz(PLAN_THREADS / n), i = tid >> lg, per = 1 << lg, j0 = tid & (per - 1);
    const int log_ps = 31 - __clz(c.ps);
    int *row = c.table + (size_t)(i < n ? sh_seq[i] : 0) * c.max_pages;
    if (i < n) {
        const int at = (sh_len[i] + c.ps - 1) >> log_ps;
        for (int j = j0; j < sh_k[i]; j += per) {
            const int p = pl.free_ids[sh_at[i] + j];
            c.ref[p] = 1;
            row[at + j] = p;
        }
    }
    __syncthreads();
    if (i < n)
        for (int j = j0; j < n_new; j += per) {
            const int at = sh_len[i] + j;
            slots[(size_t)i * n_new + j] = (row[at >> log_ps] << log_ps) + (at & (c.ps - 1));
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

// most: pages the plan may have listed.  The grid follows it up to 64 CTAs a
// SM (8 resident at a time): the later CTAs' loads of the copy list overlap the
// earlier ones' copies (1.47 GB of moves: 232 us, 6.3 TB/s with the plan; 250
// at 8 CTAs a SM, all resident).
static cudaError_t launch_copy(const xc_kv_cache &c, const KvPlan &pl, long long most, long long n_entries,
                               cudaStream_t st) {
    const int row_vecs = (int)(kv_row_bytes(c) / 16);
    const long long chunks = most * c.n_layers * 2 * (((long long)c.page_size * row_vecs + COPY_VECS - 1) / COPY_VECS);
    const long long ctas = std::max(std::min(chunks, (long long)device_sms() * 64), 1ll);
    return launch_pdl(kv_copy_kernel, dim3((unsigned)ctas), dim3(256), 0, st, reinterpret_cast<uint4 *>(c.k),
                      reinterpret_cast<uint4 *>(c.v), c.n_layers, c.n_pages, c.page_size, row_vecs, pl, c.table, n_entries);
}

cudaError_t kv_fork(const xc_kv_cache &c, int n, const int *src, const int *dst, void *ws, int *err, cudaStream_t st) {
    const KvPlan pl = kv_plan(c, ws);
    cudaError_t e = launch_pdl(kv_fork_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, kv_state(c), n, src, dst, pl, err);
    if (e != cudaSuccess) return e;
    return launch_copy(c, pl, n, 0, st);
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
    return launch_copy(c, pl, (c.n_pages + 1) / 2, (long long)c.max_seqs * c.max_pages, st);
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
