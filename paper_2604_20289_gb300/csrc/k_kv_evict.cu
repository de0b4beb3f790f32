// Eviction from the paged cache by the weight that attention gave to each token.
//
// Of a sequence longer than `keep` tokens there stay the first n_first, the last
// n_last and, between them, those of the largest weights (the lowest index first
// among equal ones), in their order.  Three kernels: a CTA per sequence picks the
// tokens, one CTA plans the pages of all of them and a third kernel moves the rows.
//
// The rows move within the sequence's own pages: kept row i comes from row idx[i]
// >= i, so a CTA that goes up the rows of one column slice in batches overwrites
// only rows that it has read, whatever the pages hold, and a full pool needs
// no spare room.  A page that other sequences hold is replaced by a fresh one
// where its rows change or it ends up partly filled, and left as it is.
#include <algorithm>
#include <climits>

#include "xc_branch.cuh"
#include "xc_pages.cuh"

namespace xc {

struct EvictPick {
    int seq, len, same, what;   // same: rows that stay where they are (idx[i] = i up to there)
};
enum { EVICT_BAD = 1, EVICT_LONG = 2 };

struct EvictSched {
    KvState c;
    int n, keep, first, last;
    const int *seqs;
    float *w;
    long w_ld;
    int *idx;                   // [n][keep] kept tokens, ascending
    EvictPick *pick;            // [n]
    int *go;                    // the plan has gone through
    int *free_ids;              // [n_pages]
    int *old;                   // [n][max_pages] pages before the call, from the first changed one; EVICT_COPIED: replaced
    int write_kept;             // idx is the caller's
};
constexpr int EVICT_COPIED = INT_MIN;

// First page of a sequence that changes, of the ceil(keep / ps) that stay.
__device__ __forceinline__ int evict_page0(const EvictSched &s, int same) {
    return same < s.keep ? same / s.c.ps : s.keep / s.c.ps;    // a last page that ends inside counts, a full one does not
}

// ------------------------------------------------------------------ selection
// Order of the weights as whole numbers: NaN below everything, -0 equal to 0.
__device__ __forceinline__ unsigned weight_key(float w) {
    if (w != w) return 0;
    const unsigned u = __float_as_uint(w + 0.0f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

constexpr int PICK_THREADS = 1024, PICK_WARPS = PICK_THREADS / 32, PICK_REGS = 8, RANK_MAX = 512;
static_assert(RANK_MAX <= PICK_THREADS && RANK_MAX % 16 == 0, "a candidate a thread");

// A warp holds a contiguous run of the candidates, 32 at a time.  The smallest
// kept key is found digit by digit, 4 bits at a time from the top: every thread counts
// its keys' digits in 8-bit fields, so no atomics and no shared histogram, warp d adds up digit d and
// every warp finds the digit by itself.  Latency bound: 8 rounds of two barriers.
// Up to 512 candidates each is compared with all others instead, four lanes a candidate:
// one pass, work with the square of the count (whole call, 16 short rows of 70, 490 and 990
// candidates: 14.2, 18.9 and 32.5 us against 22.4, 23.0 and 23.8 by digits).
__global__ void __launch_bounds__(PICK_THREADS) kv_evict_pick_kernel(const __grid_constant__ EvictSched s, int *err) {
    pdl_wait();
    pdl_release();
    __shared__ unsigned sh_digits[16][PICK_WARPS + 1];
    __shared__ __align__(16) unsigned sh_total[16];
    __shared__ __align__(16) unsigned sh_key[RANK_MAX];
    __shared__ unsigned long long sh_low[PICK_WARPS];
    __shared__ int sh_gt[PICK_WARPS], sh_eq[PICK_WARPS];
    __shared__ int sh_drop;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i = blockIdx.x;
    const int seq = s.seqs[i];
    bool bad = seq < 0 || seq >= s.c.max_seqs;
    int len = 0;
    if (!bad) {
        len = s.c.len[seq];
        bad = len < 0 || (long long)len > (long long)s.c.max_pages * s.c.ps;
    }
    if (!bad) {
        for (int j = tid; j < i; j += PICK_THREADS) bad = bad || s.seqs[j] == seq;
        const int np = (len + s.c.ps - 1) / s.c.ps;
        const int *row = s.c.table + (size_t)seq * s.c.max_pages;
        if (len > s.keep)
            for (int j = tid; j < np; j += PICK_THREADS) bad = bad || row[j] < 0 || row[j] >= s.c.n_pages;
    }
    const int cand = len - s.first - s.last, take = s.keep - s.first - s.last;     // (take < cand where the sequence is long)
    const bool search = !bad && len > s.keep && take > 0;
    const float *w = s.w + (size_t)(search ? seq : 0) * s.w_ld + s.first;
    const int seg = (cand + PICK_THREADS - 1) / PICK_THREADS * 32, c0 = warp * seg, c1 = min(c0 + seg, cand);
    float raw[PICK_REGS];
#pragma unroll
    for (int r = 0; r < PICK_REGS; ++r) raw[r] = search && c0 + 32 * r + lane < c1 ? w[c0 + 32 * r + lane] : 0.0f;
    bad = __syncthreads_or(bad);
    int *idx = s.idx + (size_t)i * s.keep;
    if (bad || len <= s.keep) {
        if (tid == 0) {
            s.pick[i] = EvictPick{seq, len, s.keep, bad ? EVICT_BAD : 0};
            if (bad && err) atomicOr(err, ERR_BAD_SEQ);
        }
        if (s.write_kept)
            for (int j = tid; j < s.keep; j += PICK_THREADS) idx[j] = j < len ? j : -1;
        return;
    }
    for (int j = tid; j < s.first; j += PICK_THREADS) idx[j] = j;
    for (int j = tid; j < s.last; j += PICK_THREADS) idx[s.keep - s.last + j] = len - s.last + j;
    if (tid == 0) sh_drop = INT_MAX;
    if (take == 0) {
        if (tid == 0) s.pick[i] = EvictPick{seq, len, min(s.first, s.keep), EVICT_LONG};
        return;
    }
    unsigned key[PICK_REGS];
#pragma unroll
    for (int r = 0; r < PICK_REGS; ++r) key[r] = c0 + 32 * r + lane < c1 ? weight_key(raw[r]) : 0;
    auto at = [&](int c) { return weight_key(w[c]); };
    unsigned top = 0, mask = 0, rest = take;           // the smallest kept key begins with top; rest: kept ones among those that do
    if (cand <= RANK_MAX) {
        // few candidates: each counts the larger ones; the threshold is the smallest with fewer than take
        if (c0 + lane < c1) sh_key[c0 + lane] = key[0];
        const int n16 = (cand + 15) / 16;
        if (tid < 16 * n16 - cand) sh_key[cand + tid] = 0;
        __syncthreads();
        unsigned long long low = ~0ull;                // (key, larger ones)
        for (int g = 0; g < cand; g += PICK_THREADS / 4) {          // four lanes a candidate
            const int c = g + (tid >> 2);
            if (g + warp * 8 >= cand) break;
            const unsigned mine = sh_key[min(c, RANK_MAX - 1)];
            unsigned larger = 0;
            for (int j = 0; j < n16; ++j) {
                const uint4 k = *reinterpret_cast<const uint4 *>(sh_key + 16 * j + 4 * (lane & 3));
                larger += (k.x > mine) + (k.y > mine) + (k.z > mine) + (k.w > mine);
            }
            larger += __shfl_xor_sync(0xffffffffu, larger, 1);
            larger += __shfl_xor_sync(0xffffffffu, larger, 2);
            if (c < cand && larger < (unsigned)take) low = min(low, (unsigned long long)mine << 32 | larger);
        }
        const unsigned k = __reduce_min_sync(0xffffffffu, (unsigned)(low >> 32));
        const unsigned l = __reduce_min_sync(0xffffffffu, (unsigned)(low >> 32) == k ? (unsigned)low : ~0u);
        if (lane == 0) sh_low[warp] = (unsigned long long)k << 32 | l;
        __syncthreads();
        low = sh_low[lane];
        top = __reduce_min_sync(0xffffffffu, (unsigned)(low >> 32));
        rest = take - __reduce_min_sync(0xffffffffu, (unsigned)(low >> 32) == top ? (unsigned)low : ~0u);
    } else for (int shift = 28; shift >= 0; shift -= 4) {
        unsigned long long n0 = 0, n1 = 0;             // counts of digits 0-7 and 8-15
        unsigned sum[8] = {};
        auto count = [&](unsigned k) {
            if ((k & mask) == top) {
                const unsigned d = (k >> shift) & 15;
                const unsigned long long one = 1ull << (8 * (d & 7));
                n0 += d < 8 ? one : 0;
                n1 += d < 8 ? 0 : one;
            }
        };
        auto spill = [&]() {                           // 8-bit fields into 16-bit pairs, over the warp
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned a = (unsigned)(n0 >> (16 * j)) & 0xffffu, b = (unsigned)(n1 >> (16 * j)) & 0xffffu;
                sum[j] += __reduce_add_sync(0xffffffffu, (a & 0xffu) | (a >> 8) << 16);
                sum[4 + j] += __reduce_add_sync(0xffffffffu, (b & 0xffu) | (b >> 8) << 16);
            }
            n0 = n1 = 0;
        };
#pragma unroll
        for (int r = 0; r < PICK_REGS; ++r)
            if (c0 + 32 * r + lane < c1) count(key[r]);
        // rows of more than 8192 candidates read the others again; a pair's 16 bits hold 65535 of a warp's
        unsigned wide[16];
        const bool many = seg > 32 * PICK_REGS;
        spill();
        if (many) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                wide[2 * j] = sum[j] & 0xffffu;
                wide[2 * j + 1] = sum[j] >> 16;
                sum[j] = 0;
            }
            for (int b0 = c0 + 32 * PICK_REGS; b0 < c1; b0 += 32 * 128) {
                const int b1 = min(b0 + 32 * 128, c1);
                for (int c = b0 + lane; c < b1; c += 32) count(at(c));
                __syncwarp();
                spill();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    wide[2 * j] += sum[j] & 0xffffu;
                    wide[2 * j + 1] += sum[j] >> 16;
                    sum[j] = 0;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                wide[2 * j] = sum[j] & 0xffffu;
                wide[2 * j + 1] = sum[j] >> 16;
            }
        }
        // digit d's total over the warps: warp d adds it up
        unsigned mine = 0;
#pragma unroll
        for (int d = 0; d < 16; ++d)
            if (lane == d) mine = wide[d];
        if (lane < 16) sh_digits[lane][warp] = mine;
        __syncthreads();
        if (warp < 16) {
            const unsigned t = __reduce_add_sync(0xffffffffu, sh_digits[warp][lane]);
            if (lane == 0) sh_total[warp] = t;
        }
        __syncthreads();
        const unsigned t = sh_total[lane & 15];        // keys of this digit or a larger one, in lane `digit`
        unsigned ge = lane < 16 ? t : 0;
#pragma unroll
        for (int d = 1; d < 16; d *= 2) ge += __shfl_down_sync(0xffffffffu, ge, d);
        const unsigned digit = 31 - __clz(__ballot_sync(0xffffffffu, lane < 16 && ge >= rest));
        const unsigned above = __shfl_sync(0xffffffffu, ge - t, digit);
        top |= digit << shift;
        mask |= 15u << shift;
        rest -= above;
    }
    // keys above top all stay, and the first `rest` of those equal to it
    int gt = 0, eq = 0;
    auto each = [&](auto &&f) {                        // every candidate of the warp, 32 at a time; converged
#pragma unroll
        for (int r = 0; r < PICK_REGS; ++r)
            if (c0 + 32 * r < c1) f(c0 + 32 * r + lane, key[r]);
        for (int c = c0 + 32 * PICK_REGS; c < c1; c += 32) f(c + lane, c + lane < c1 ? at(c + lane) : 0u);
    };
    each([&](int c, unsigned k) {
        const bool in = c < c1;
        gt += __popc(__ballot_sync(0xffffffffu, in && k > top));
        eq += __popc(__ballot_sync(0xffffffffu, in && k == top));
    });
    if (lane == 0) {
        sh_gt[warp] = gt;
        sh_eq[warp] = eq;
    }
    __syncthreads();
    int gt0 = 0, eq0 = 0;
    for (int v = 0; v < warp; ++v) {
        gt0 += sh_gt[v];
        eq0 += sh_eq[v];
    }
    int out = s.first + gt0 + min(eq0, (int)rest), drop = INT_MAX;
    const unsigned below = (1u << lane) - 1;
    each([&](int c, unsigned k) {
        const bool in = c < c1;
        const unsigned same = __ballot_sync(0xffffffffu, in && k == top);
        const bool stay = in && (k > top || (k == top && eq0 + __popc(same & below) < (int)rest));
        const unsigned kept = __ballot_sync(0xffffffffu, stay);
        if (stay) idx[out + __popc(kept & below)] = s.first + c;
        else if (in) drop = min(drop, s.first + c);
        eq0 += __popc(same);
        out += __popc(kept);
    });
    drop = __reduce_min_sync(0xffffffffu, drop);
    if (lane == 0 && drop != INT_MAX) atomicMin(&sh_drop, drop);
    __syncthreads();
    if (tid == 0) s.pick[i] = EvictPick{seq, len, min(sh_drop, s.keep), EVICT_LONG};
}

// --------------------------------------------------------------------- pages
// A warp per sequence.  What each page becomes is settled before anything changes: sequences
// of one call may hold the same page.
__global__ void __launch_bounds__(PLAN_THREADS) kv_evict_plan_kernel(const __grid_constant__ EvictSched s, int *err) {
    pdl_wait();
    pdl_release();
    __shared__ int sh[32], sh_need[PLAN_THREADS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const KvState &c = s.c;
    const bool bad = tid < s.n && (s.pick[tid].what & EVICT_BAD) != 0;
    if (tid == 0) *s.go = 0;
    if (__syncthreads_or(bad)) return;                 // flagged already
    const int stay = (s.keep + c.ps - 1) / c.ps;
    sh_need[tid] = 0;
    __syncthreads();
    for (int i = warp; i < s.n; i += 32) {
        const EvictPick p = s.pick[i];
        if ((p.what & EVICT_LONG) == 0) continue;
        const int np = (p.len + c.ps - 1) / c.ps, p0 = evict_page0(s, p.same);
        const int *row = c.table + (size_t)p.seq * c.max_pages;
        int *old = s.old + (size_t)i * c.max_pages;
        int need = 0;
        for (int j0 = p0; j0 < np; j0 += 32) {
            const int j = j0 + lane;
            const int id = j < np ? row[j] : 0;
            const bool copy = j < stay && j < np && c.ref[id] > 1;
            if (j < np) old[j] = copy ? id | EVICT_COPIED : id;
            need += __popc(__ballot_sync(0xffffffffu, copy));
        }
        if (lane == 0) sh_need[i] = need;
    }
    __syncthreads();
    int need;
    const int at = block_scan(sh_need[tid], sh, need);
    __syncthreads();
    sh_need[tid] = at;
    const int found = list_pages(c.ref, 0, c.n_pages, false, need, s.free_ids, sh);
    if (found < need) {
        if (tid == 0 && err) atomicOr(err, ERR_CACHE_FULL);
        return;
    }
    for (int i = warp; i < s.n; i += 32) {
        const EvictPick p = s.pick[i];
        if ((p.what & EVICT_LONG) == 0) continue;
        const int np = (p.len + c.ps - 1) / c.ps, p0 = evict_page0(s, p.same);
        int *row = c.table + (size_t)p.seq * c.max_pages;
        const int *old = s.old + (size_t)i * c.max_pages;
        int next = sh_need[i];
        for (int j0 = p0; j0 < np; j0 += 32) {
            const int j = j0 + lane;
            const int id = j < np ? old[j] : 0;
            const bool copy = j < np && id < 0;
            const unsigned mask = __ballot_sync(0xffffffffu, copy);
            if (copy) {
                const int fresh = s.free_ids[next + __popc(mask & ((1u << lane) - 1))];
                c.ref[fresh] = 1;
                row[j] = fresh;
                atomicSub(&c.ref[id & INT_MAX], 1);
            } else if (j >= stay && j < np) {
                row[j] = -1;
                atomicSub(&c.ref[id], 1);
            }
            next += __popc(mask);
        }
        if (lane == 0) c.len[p.seq] = s.keep;
    }
    if (tid == 0) *s.go = 1;
}

// ---------------------------------------------------------------------- rows
// An item is a column slice of SV 16-byte vectors of one sequence's keys or values
// in one layer, or its weights.  Batches of UN x (256 / SV) rows: loads, a barrier,
// stores.  The next batch's loads need not wait for the stores, whose rows lie below
// everything that is still to be read.  HBM bound: 6 branches of 2000..2977 tokens to 2003, 30 layers of 12 x 128, 6.5 TB/s.
constexpr int MOVE_THREADS = 256, MOVE_UN = 8;
__global__ void __launch_bounds__(MOVE_THREADS)
    kv_evict_move_kernel(uint4 *k, uint4 *v, const int n_layers, const int row_vecs, const int log_sv,
                         const __grid_constant__ EvictSched s) {
    pdl_wait();
    pdl_release();
    const KvState &c = s.c;
    const int go = *s.go, tid = threadIdx.x;
    if (!go) {                                         // nothing has changed
        if (s.write_kept)
            for (long x = (long)blockIdx.x * MOVE_THREADS + tid; x < (long)s.n * s.keep; x += (long)gridDim.x * MOVE_THREADS) s.idx[x] = -1;
        return;
    }
    const int log_ps = 31 - __clz(c.ps), sv = 1 << log_sv, slices = (row_vecs + sv - 1) >> log_sv;
    const int per = MOVE_THREADS >> log_sv, lane = tid & (sv - 1), r_in = tid >> log_sv;
    const long n_w = s.w != nullptr ? s.n : 0, total = n_w + (long)s.n * n_layers * 2 * slices;
    for (long it = blockIdx.x; it < total; it += gridDim.x) {
        const bool weights = it < n_w;
        const long x = weights ? it : it - n_w;
        const int i = (int)(x % s.n);
        const EvictPick p = s.pick[i];
        if ((p.what & EVICT_LONG) == 0) continue;
        const int *idx = s.idx + (size_t)i * s.keep;
        if (weights) {
            float *w = s.w + (size_t)p.seq * s.w_ld;
            for (int b0 = p.same; b0 < s.keep; b0 += MOVE_UN * MOVE_THREADS) {
                float t[MOVE_UN];
#pragma unroll
                for (int u = 0; u < MOVE_UN; ++u) {
                    const int r = b0 + u * MOVE_THREADS + tid;
                    if (r < s.keep) t[u] = w[idx[r]];
                }
                __syncthreads();
#pragma unroll
                for (int u = 0; u < MOVE_UN; ++u) {
                    const int r = b0 + u * MOVE_THREADS + tid;
                    if (r < s.keep) w[r] = t[u];
                }
            }
            __syncthreads();                           // every weight has been read
            for (int r = s.keep + tid; r < p.len; r += MOVE_THREADS) w[r] = 0.0f;
            continue;
        }
        const int lk = (int)(x / s.n), slice = lk % slices, layer = lk / slices >> 1;
        uint4 *pool = ((lk / slices) & 1 ? v : k) + (size_t)layer * c.n_pages * c.ps * row_vecs;
        const int col = (slice << log_sv) + lane;
        const int *old = s.old + (size_t)i * c.max_pages, *row = c.table + (size_t)p.seq * c.max_pages;
        const int p0 = evict_page0(s, p.same);
        int r0 = p.same;                               // a replaced page takes its unchanged rows along
        if (p0 * c.ps < s.keep && old[p0] < 0) r0 = p0 << log_ps;
        for (int b0 = r0; b0 < s.keep; b0 += MOVE_UN * per) {
            uint4 t[MOVE_UN];
#pragma unroll
            for (int u = 0; u < MOVE_UN; ++u) {
                const int r = b0 + u * per + r_in;
                if (r < s.keep && col < row_vecs) {
                    const int from = idx[r];
                    const size_t at = ((size_t)(old[from >> log_ps] & INT_MAX) << log_ps) + (from & (c.ps - 1));
                    t[u] = __ldcs(pool + at * row_vecs + col);
                }
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < MOVE_UN; ++u) {
                const int r = b0 + u * per + r_in;
                if (r < s.keep && col < row_vecs) {
                    const size_t at = ((size_t)row[r >> log_ps] << log_ps) + (r & (c.ps - 1));
                    __stcs(pool + at * row_vecs + col, t[u]);
                }
            }
        }
    }
}

// ------------------------------------------------------------------- host
static size_t evict_ints(const xc_kv_cache &c, int n, int keep) {
    return 4 + 4 * (size_t)n + c.n_pages + (size_t)n * c.max_pages + (size_t)n * keep;
}
size_t kv_evict_workspace_bytes(const xc_kv_cache &c, int n, int keep) { return evict_ints(c, n, keep) * sizeof(int); }

cudaError_t kv_evict(const xc_kv_cache &c, int n, const int *seqs, int keep, int n_first, int n_last, float *weights, long w_ld,
                     int *kept, void *ws, int *err, cudaStream_t st) {
    EvictSched s{};
    s.c = kv_state(c);
    s.n = n;
    s.keep = keep;
    s.first = n_first;
    s.last = n_last;
    s.seqs = seqs;
    s.w = weights;
    s.w_ld = w_ld;
    int *p = reinterpret_cast<int *>(ws);
    s.go = p;
    s.pick = reinterpret_cast<EvictPick *>(p + 4);
    s.free_ids = p + 4 + 4 * (size_t)n;
    s.old = s.free_ids + c.n_pages;
    s.idx = kept != nullptr ? kept : s.old + (size_t)n * c.max_pages;
    s.write_kept = kept != nullptr;
    cudaError_t e = launch_pdl(kv_evict_pick_kernel, dim3(n), dim3(PICK_THREADS), 0, st, s, err);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kv_evict_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, s, err);
    if (e != cudaSuccess) return e;
    const int row_vecs = (int)(kv_row_bytes(c) / 16), sms = device_sms();
    int log_sv = 5;                                    // 512 bytes of a row, less where there are few slices
    while (log_sv > 2 && ((1 << log_sv) > row_vecs || (long)n * c.n_layers * 2 * ((row_vecs + (1 << log_sv) - 1) >> log_sv) < 8l * sms)) --log_sv;
    const long items = (long)n * c.n_layers * 2 * ((row_vecs + (1 << log_sv) - 1) >> log_sv) + n;
    const unsigned ctas = (unsigned)std::min(items, 64l * sms);
    return launch_pdl(kv_evict_move_kernel, dim3(ctas), dim3(MOVE_THREADS), 0, st, reinterpret_cast<uint4 *>(c.k),
                      reinterpret_cast<uint4 *>(c.v), c.n_layers, row_vecs, log_sv, s);
}

}  // namespace xc
