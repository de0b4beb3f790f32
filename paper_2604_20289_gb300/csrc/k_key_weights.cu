// The weight that attention gave to each cached key.
//
//   w[s][j] = decay w[s][j] + sum_{i, h} exp(scale q_ih . k_j - lse_ih),
//
// over the query rows (token i, head h) that see key j; lse is the log of a
// row's sum of exponentials, which the attention leaves, so that one pass over
// the keys is enough.  The scores are computed as S^T = K Q^T: a key is a row of
// the product and a lane of tensor memory, so the sum over the query rows stays
// in one thread's registers.
//
// A unit is (128 keys, the rows that are summed for them), its steps the unit's key
// heads x row tiles.  All units' steps form one line that the CTAs share evenly, as
// in the attention: a unit that one CTA runs whole is written at once, the sums
// of a cut one leave as partials that key_merge_kernel adds in CTA order, so a call
// gives the same bits every time.  Where every branch has few rows and the
// branches share keys, a unit of shared keys takes the rows of as many branches
// as fit a row tile (packed): the keys are read once for all of them, and every
// column's sum is kept apart until the unit's end.
#include <algorithm>

#include "xc_branch.cuh"
#include "xc_ptx.cuh"

namespace xc {

constexpr int KW_MAX_B = 1024;           // branches of a call
constexpr int KW_KEYS = 128, KW_COLS = 128, KW_BUFS = 4;
constexpr int KW_SWAPS = 2 * KW_BUFS;   // pieces of a step each that one half of the threads may be ahead of the other, and more
constexpr float KW_LOG2E = 1.4426950408889634f;

struct KeySched {
    int B, n_q, grp, Hk, causal, G;
    int max_seqs, max_pages, ps, n_pages, shared;
    int P, n_pt;             // keys and key tiles of the packed shared units (0: none)
    int packed;              // a row tile holds branches' rows side by side; else one branch's
    int tt, N, n_ct;         // tokens and columns of a row tile; row tiles (of all rows if packed, else of a branch)
    int nb;                  // branches of a row tile at most
    float decay, sl2;
    const int *seqs, *len, *table;
    const float *lse;        // [B n_q][Hk grp]
    float *w;
    long w_ld;
    int4 *meta;              // [2 G] what a CTA's cut pieces are
    float *part;             // [2 G][nb][128]

    __device__ __forceinline__ int limit(int l, int i) const { return causal ? l - n_q + i + 1 : l; }
};
enum { KW_CUT = 1, KW_BEGIN = 2, KW_END = 4 };

// Lengths and sequences of the branches, and the line.  A sequence out of range, of an
// impossible length, or listed before has length 0 and takes no part.
struct KeyLens {
    int len[KW_MAX_B], seq[KW_MAX_B], off[KW_MAX_B + 1];
    int scan[32];
};

template <int KT>
__device__ __forceinline__ int key_tiles(const KeySched &s, int l) {
    return l > s.P ? (l - s.P + KT - 1) / KT : 0;
}
// First row tile that sees the own tile kt of a branch of length l.
template <int KT>
__device__ __forceinline__ int key_first_ct(const KeySched &s, int l, int kt) {
    if (s.packed || !s.causal) return 0;
    const int i0 = kt * KT - (l - s.n_q);
    return i0 > 0 ? i0 / s.tt : 0;
}
template <int KT>
__device__ __forceinline__ int key_steps(const KeySched &s, int l, int kt) {
    return s.Hk * ((s.packed ? 1 : s.n_ct) - key_first_ct<KT>(s, l, kt));
}
template <int KT>
__device__ int key_full_tiles(const KeySched &s, int l) {      // own tiles that every row tile sees
    const int n = key_tiles<KT>(s, l);
    if (s.packed || !s.causal) return n;
    return l < s.n_q ? 0 : min(n, (l - s.n_q) / KT + 1);
}

// Every thread calls it.  line: whether the scan of the steps is wanted too.
template <int KT>
__device__ void key_lens(const KeySched &s, KeyLens &L, int *err) {
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int b = tid; b < s.B; b += nt) L.seq[b] = s.seqs[b];
    __syncthreads();
    bool bad = false;
    for (int b = tid; b < s.B; b += nt) {
        const int q = L.seq[b];
        int l = 0;
        if (q >= 0 && q < s.max_seqs) {
            l = s.len[q];
            bool wrong = l < 0 || l > s.max_pages * s.ps;
            bad = bad || l < s.shared;
            for (int j = 0; j < b; ++j) wrong = wrong || L.seq[j] == q;
            if (wrong) {
                bad = true;
                l = 0;
            }
        } else {
            bad = true;
        }
        L.len[b] = l;
    }
    if (bad && err && blockIdx.x == 0) atomicOr(err, ERR_BAD_SEQ);
    __syncthreads();
    // steps of each branch's own tiles: exclusive scan
    const int per = (s.B + nt - 1) / nt, b0 = min(tid * per, s.B), b1 = min(b0 + per, s.B);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int l = L.len[b], n = key_tiles<KT>(s, l), full = key_full_tiles<KT>(s, l);
        int x = full * s.Hk * (s.packed ? 1 : s.n_ct);
        for (int kt = full; kt < n; ++kt) x += key_steps<KT>(s, l, kt);
        L.off[b + 1] = x;
        mine += x;
    }
    int x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) L.scan[warp] = x;
    __syncthreads();
    int before = x - mine;
    for (int w = 0; w < warp; ++w) before += L.scan[w];
    if (tid == 0) L.off[0] = 0;
    for (int b = b0; b < b1; ++b) {
        before += L.off[b + 1];
        L.off[b + 1] = before;
    }
    __syncthreads();
}

struct KeyPiece {
    int own, b;              // own tile of branch b, or shared tile
    int kt, key0;            // tile and its first key
    int t0, ct0, nct;        // first token of row tile ct0; row tiles
    int s0, s1, n;           // steps of the piece, of the unit
};
struct KeyWalk {
    int own, b, kt, ct, off, left;
    template <int KT>
    __device__ __forceinline__ void start(const KeySched &s, const KeyLens &L, int c) {
        const unsigned pp = (unsigned)s.n_pt * s.n_ct * s.Hk, T = pp + L.off[s.B];
        const unsigned q = T / s.G, r = T - q * s.G;
        unsigned x = q * c + min((unsigned)c, r);
        left = q + ((unsigned)c < r ? 1 : 0);
        own = b = kt = ct = off = 0;
        if (left == 0) return;
        if (x < pp) {
            const int u = x / s.Hk;
            off = x - u * s.Hk;
            kt = u / s.n_ct;
            ct = u - kt * s.n_ct;
            return;
        }
        x -= pp;
        own = 1;
        int lo = 0, hi = s.B;                          // the last b with off[b] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((unsigned)L.off[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo;
        int rest = x - L.off[b];
        const int l = L.len[b], each = s.Hk * (s.packed ? 1 : s.n_ct), full = key_full_tiles<KT>(s, l);
        if (rest < full * each) {
            kt = rest / each;
            off = rest - kt * each;
            return;
        }
        rest -= full * each;
        for (kt = full;; ++kt) {
            const int n = key_steps<KT>(s, l, kt);
            if (rest < n) break;
            rest -= n;
        }
        off = rest;
    }
    template <int KT>
    __device__ __forceinline__ bool next(const KeySched &s, const KeyLens &L, KeyPiece &p) {
        while (left > 0) {
            if (!own && kt == s.n_pt) {                // (n_pt = 0 too)
                own = 1;
                b = kt = off = 0;
            }
            if (!own) {
                p.n = s.Hk;
                p.ct0 = ct;
                p.t0 = ct * s.tt;
                p.key0 = kt * KT;
                p.nct = 1;
            } else {
                while (kt >= key_tiles<KT>(s, L.len[b])) {
                    ++b;
                    kt = 0;
                }
                p.n = key_steps<KT>(s, L.len[b], kt);
                p.ct0 = key_first_ct<KT>(s, L.len[b], kt);
                p.t0 = b * s.n_q + p.ct0 * s.tt;
                p.key0 = s.P + kt * KT;
                p.nct = (s.packed ? 1 : s.n_ct) - p.ct0;
            }
            p.own = own;
            p.b = b;
            p.kt = kt;
            p.s0 = off;
            p.s1 = min(p.n, off + left);
            left -= p.s1 - p.s0;
            off = 0;
            if (own || ++ct == s.n_ct) {
                ct = 0;
                ++kt;
            }
            return true;
        }
        return false;
    }
};

// ------------------------------------------------------- tensor-core kernel
// Warps: 0 loads (key tiles page by page, row tiles), 1 issues the products, 2 reads
// the rows' lse and limits, 4-11 take the exponentials (thread = key, two per TMEM
// quadrant, half of the columns each).
constexpr int KW_THREADS = 384;
struct KeyRing {
    int ks, qs;              // slots of key tiles, of row tiles
};
struct alignas(16) KeyCols {           // what a step's columns need
    float nl[KW_COLS];       // -lse log2(e)
    int lim[KW_COLS];        // keys of the tile that the column's row sees
    int masked;
};

template <int HD, bool PACKED>
__global__ void __launch_bounds__(KW_THREADS, 1)
    key_weights_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ KeySched s, const KeyRing ring, int *err) {
    constexpr int NR = HD / 64, K_REGION = KW_KEYS * 128, K_BYTES = NR * K_REGION;
    extern __shared__ uint8_t smem_raw[];
    __shared__ KeyLens L;
    __shared__ KeyCols cols[KW_BUFS];
    __shared__ float sh_half[KW_SWAPS][KW_KEYS];
    __shared__ uint64_t bars[32 + 3 * KW_BUFS + KW_SWAPS + 1];
    __shared__ uint32_t tmem_slot;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int q_region = s.N * 128, q_bytes = NR * q_region;
    uint8_t *sK = smem, *sQ = smem + ring.ks * K_BYTES;
    uint64_t *k_full = bars, *k_empty = bars + 8, *q_full = bars + 16, *q_empty = bars + 24;
    uint64_t *s_full = bars + 32, *s_empty = s_full + KW_BUFS, *l_full = s_empty + KW_BUFS;
    uint64_t *swap = l_full + KW_BUFS, *drained = swap + KW_SWAPS;   // swap: one half's sums are in sh_half
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1);
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < KW_BUFS; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 256);
            mbar_init(&l_full[i], 32);
        }
        for (int i = 0; i < KW_SWAPS; ++i) mbar_init(&swap[i], 128);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(&tmem_slot, 512);
    // columns that no row tile fills stay zero
    for (int x = threadIdx.x; x < ring.qs * q_bytes / 16; x += KW_THREADS) reinterpret_cast<uint4 *>(sQ)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    pdl_wait();
    key_lens<KW_KEYS>(s, L, err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    KeyWalk walk;
    walk.start<KW_KEYS>(s, L, blockIdx.x);
    KeyPiece p;

    if (warp == 0) {
        const int box = min(s.ps, KW_KEYS), log_ps = 31 - __clz(s.ps);
        int kc = 0, qc = 0;
        bool ok = true;
        while (ok && walk.next<KW_KEYS>(s, L, p)) {
            const int seq = L.seq[p.own ? p.b : 0];
            const bool there = seq >= 0 && seq < s.max_seqs;
            const int keys = (p.own ? L.len[p.b] : s.P) - p.key0;
            int row = -1;                              // first pool row of this lane's page of the tile
            if (lane * box < KW_KEYS && lane * box < keys) {
                const int key = p.key0 + lane * box, id = there ? s.table[(size_t)seq * s.max_pages + (key >> log_ps)] : -1;
                const bool good = id >= 0 && id < s.n_pages;
                if (!good && err) atomicOr(err, ERR_BAD_SEQ);
                row = good ? id * s.ps + (key & (s.ps - 1)) : s.n_pages * s.ps;      // out of range: TMA fills zeros
            }
            const uint32_t k_tx = __popc(__ballot_sync(0xffffffffu, row >= 0)) * box * 128 * NR;
            for (int st = p.s0; st < p.s1; ++st, ++qc) {
                const int h = PACKED ? st : st / p.nct, ct = PACKED ? 0 : st - h * p.nct;
                if (st == p.s0 || ct == 0) {
                    const int i = kc % ring.ks;
                    ok = mbar_wait(&k_empty[i], ((kc / ring.ks) & 1) ^ 1, err, ERR_WAIT_PRODUCER);
                    if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                    if (lane == 0) mbar_expect_tx(&k_full[i], k_tx);
                    __syncwarp();
                    if (row >= 0)
                        for (int r = 0; r < NR; ++r)
                            tma_load_2d(sK + i * K_BYTES + r * K_REGION + lane * box * 128, &tmK, &k_full[i], h * HD + 64 * r, row);
                    ++kc;
                }
                const int i = qc % ring.qs;
                ok = mbar_wait(&q_empty[i], ((qc / ring.qs) & 1) ^ 1, err, ERR_WAIT_PRODUCER);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                if (lane == 0) {
                    mbar_expect_tx(&q_full[i], NR * s.tt * s.grp * 128);
                    for (int r = 0; r < NR; ++r)
                        tma_load_3d(sQ + i * q_bytes + r * q_region, &tmQ, &q_full[i], 64 * r, h * s.grp, p.t0 + ct * s.tt);
                }
                __syncwarp();
            }
        }
        if (lane == 0) {                               // every copy has landed before the CTA exits
            for (int j = max(kc - ring.ks, 0); j < kc; ++j) mbar_wait(&k_full[j % ring.ks], (j / ring.ks) & 1, err, ERR_WAIT_PRODUCER);
            for (int j = max(qc - ring.qs, 0); j < qc; ++j) mbar_wait(&q_full[j % ring.qs], (j / ring.qs) & 1, err, ERR_WAIT_PRODUCER);
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_bf16(KW_KEYS, 16, false, false) - ((16u >> 3) << 17) + ((uint32_t)(s.N >> 3) << 17);
        const uint64_t dK = sdesc_sw128(smem_u32(sK), 16, 1024), dQ = sdesc_sw128(smem_u32(sQ), 16, 1024);
        auto wait = [&](uint64_t *b, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(b, parity & 1, err, ERR_WAIT_MMA)) != 0;
        };
        int kc = 0, it = 0;
        bool ok = true;
        while (ok && walk.next<KW_KEYS>(s, L, p)) {
            int ct = PACKED ? 0 : p.s0 % p.nct;
            for (int st = p.s0; st < p.s1; ++st, ++it) {
                const int ki = kc % ring.ks, qi = it % ring.qs, buf = it % KW_BUFS;
                if ((st == p.s0 || ct == 0) && !(ok = wait(&k_full[ki], kc / ring.ks))) break;
                if (!(ok = wait(&q_full[qi], it / ring.qs) && wait(&s_empty[buf], (it / KW_BUFS) ^ 1))) break;
                tc_fence_after();
                const uint64_t da = dK + (uint64_t)((ki * K_BYTES) >> 4), db = dQ + (uint64_t)((qi * q_bytes) >> 4);
#pragma unroll
                for (int k = 0; k < HD / 16; ++k)
                    tc_mma_warp(tmem + buf * KW_COLS, da + (((k >> 2) * K_REGION + (k & 3) * 32) >> 4),
                                db + (((k >> 2) * q_region + (k & 3) * 32) >> 4), idesc, k > 0 ? 1u : 0u);
                tc_commit_warp(&q_empty[qi]);
                if (++ct == p.nct) ct = 0;
                if (PACKED || ct == 0 || st + 1 == p.s1) {
                    tc_commit_warp(&k_empty[ki]);
                    ++kc;
                }
                tc_commit_warp(&s_full[buf]);
            }
        }
        if (!ok) {                                     // a wait ran out: no product is under way when the CTA ends
            tc_commit_warp(drained);
            wait(drained, 0);
        }
    } else if (warp == 2) {
        int tk[4], gq[4], it = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 32 * i;
            tk[i] = c / s.grp;
            gq[i] = c - tk[i] * s.grp;
        }
        bool ok = true;
        while (ok && walk.next<KW_KEYS>(s, L, p)) {
            for (int st = p.s0; st < p.s1; ++st, ++it) {
                const int h = PACKED ? st : st / p.nct, ct = PACKED ? 0 : st - h * p.nct;
                const int buf = it % KW_BUFS, t0 = p.t0 + ct * s.tt;
                const int t_end = p.own ? (p.b + 1) * s.n_q : s.B * s.n_q;
                float nl[4];
                int lim[4];
                bool masked = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = t0 + tk[i];
                    nl[i] = -INFINITY;
                    lim[i] = 0;
                    if (lane + 32 * i < s.N) {
                        if (tk[i] < s.tt && t < t_end) {
                            const int b = p.own ? p.b : t / s.n_q;
                            nl[i] = -KW_LOG2E * s.lse[(size_t)t * (s.Hk * s.grp) + h * s.grp + gq[i]];
                            if (nl[i] == INFINITY) nl[i] = -INFINITY;      // a row that saw no key
                            lim[i] = min(max(s.limit(L.len[b], t - b * s.n_q) - p.key0, 0), KW_KEYS);
                        }
                        masked = masked || lim[i] < KW_KEYS;
                    }
                }
                ok = mbar_wait(&s_empty[buf], ((it / KW_BUFS) & 1) ^ 1, err, ERR_WAIT_SOFTMAX);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    cols[buf].nl[lane + 32 * i] = nl[i];
                    cols[buf].lim[lane + 32 * i] = lim[i];
                }
                const unsigned any = __ballot_sync(0xffffffffu, masked);
                if (lane == 0) cols[buf].masked = any != 0;
                mbar_arrive(&l_full[buf]);
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2, r = 32 * q + lane;
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16);
        const int nc = s.N / 16, ch0 = half ? (nc + 1) / 2 : 0, ch1 = half ? nc : (nc + 1) / 2;   // this thread's columns, by 16
        if (warp == 4 && lane < 2) s.meta[2 * blockIdx.x + lane] = make_int4(0, 0, 0, 0);
        __syncwarp();
        int it = 0, np = 0;
        bool ok = true;
        while (ok && walk.next<KW_KEYS>(s, L, p)) {
            float acc[PACKED ? 64 : 1];
#pragma unroll
            for (int i = 0; i < (PACKED ? 64 : 1); ++i) acc[i] = 0.0f;
            for (int st = p.s0; st < p.s1; ++st, ++it) {
                const int buf = it % KW_BUFS;
                const uint32_t ph = (it / KW_BUFS) & 1;
                ok = mbar_wait(&l_full[buf], ph, err, ERR_WAIT_SOFTMAX) && mbar_wait(&s_full[buf], ph, err, ERR_WAIT_SOFTMAX);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                tc_fence_after();
                const bool masked = cols[buf].masked;
                float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (ch0 + k >= ch1) break;
                    const int c = 16 * (ch0 + k);
                    float x[16];
                    tmem_ld16_sync(lanes + buf * KW_COLS + c, x);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 nl = *reinterpret_cast<const float4 *>(&cols[buf].nl[c + i]);
                        const float2 a = __ffma2_rn(make_float2(x[i], x[i + 1]), make_float2(s.sl2, s.sl2), make_float2(nl.x, nl.y));
                        const float2 b = __ffma2_rn(make_float2(x[i + 2], x[i + 3]), make_float2(s.sl2, s.sl2), make_float2(nl.z, nl.w));
                        x[i] = exp2_mufu(a.x);
                        x[i + 1] = exp2_mufu(a.y);
                        x[i + 2] = exp2_mufu(b.x);
                        x[i + 3] = exp2_mufu(b.y);
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const int4 lim = *reinterpret_cast<const int4 *>(&cols[buf].lim[c + i]);
                            if (r >= lim.x) x[i] = 0.0f;
                            if (r >= lim.y) x[i + 1] = 0.0f;
                            if (r >= lim.z) x[i + 2] = 0.0f;
                            if (r >= lim.w) x[i + 3] = 0.0f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        if constexpr (PACKED) {
                            acc[16 * k + i] += x[i];
                            acc[16 * k + i + 1] += x[i + 1];
                        } else {
                            sum = __fadd2_rn(sum, make_float2(x[i], x[i + 1]));
                        }
                    }
                }
                if constexpr (!PACKED) acc[0] += sum.x + sum.y;
                tc_fence_before();
                mbar_arrive(&s_empty[buf]);
            }
            if (!ok) break;
            const bool whole = p.s1 - p.s0 == p.n;
            const int slot = 2 * blockIdx.x + (np == 0 ? 0 : 1), key = p.key0 + r;
            if (!whole && warp == 4 && lane == 0)
                s.meta[slot] = make_int4(KW_CUT | (p.s0 == 0 ? KW_BEGIN : 0) | (p.s1 == p.n ? KW_END : 0), p.own ? p.b : -1 - p.ct0, p.key0, p.own ? 0x7fffffff : s.P);
            const int bfirst = p.own ? p.b : p.t0 / s.n_q;
            auto put = [&](int b, float v) {
                if (!p.own && key >= s.P) return;
                if (!whole) {
                    s.part[((size_t)slot * s.nb + b - bfirst) * KW_KEYS + r] = v;
                } else if (key < L.len[b]) {
                    float *at = s.w + (size_t)L.seq[b] * s.w_ld + key;
                    *at = s.decay == 0.0f ? v : fmaf(s.decay, *at, v);
                }
            };
            const int sw = np % KW_SWAPS;
            float *other = sh_half[sw];
            auto take = [&]() -> bool {                // the other half's sums
                return __all_sync(0xffffffffu, mbar_wait(&swap[sw], (np / KW_SWAPS) & 1, err, ERR_WAIT_SOFTMAX)) != 0;
            };
            if constexpr (!PACKED) {
                if (half == 1) {
                    other[r] = acc[0];
                    mbar_arrive(&swap[sw]);
                } else {
                    if (!(ok = take())) break;
                    put(p.b, acc[0] + other[r]);
                }
            } else {
                // this thread's columns, branch by branch; one branch may lie in both halves
                const int each = s.n_q * s.grp;
                const int ncol = min(p.own ? each : (s.B * s.n_q - p.t0) * s.grp, s.tt * s.grp);
                const int mid = 16 * ((nc + 1) / 2);
                auto run = [&](int c0, int c1) {
                    int b = bfirst, end = p.own ? each : ((b + 1) * s.n_q - p.t0) * s.grp;   // the column behind branch b
                    while (end <= c0) {
                        end += each;
                        ++b;
                    }
                    float v = half == 1 && c0 < ncol && end - each < mid ? other[r] : 0.0f;
#pragma unroll
                    for (int i = 0; i < 64; ++i) {
                        if (c0 + i < c1) {
                            v += acc[i];
                            if (c0 + i + 1 == min(end, ncol)) {
                                put(b, v);
                                v = 0.0f;
                                end += each;
                                ++b;
                            }
                        }
                    }
                    if (half == 0) other[r] = v;
                };
                if (half == 0) {
                    run(0, min(mid, ncol));
                    mbar_arrive(&swap[sw]);
                } else {
                    if (!(ok = take())) break;
                    run(mid, ncol);
                }
            }
            ++np;
        }
    }
    pdl_release();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Adds the pieces of a cut unit in CTA order.  grid: (slots, branches of a row tile).
__global__ void __launch_bounds__(KW_KEYS) key_merge_kernel(const __grid_constant__ KeySched s) {
    pdl_wait();
    pdl_release();
    const int4 m = s.meta[blockIdx.x];
    if ((m.x & KW_CUT) == 0 || (m.x & KW_BEGIN) == 0) return;
    int b = m.y;
    if (m.y < 0) {
        b = (-1 - m.y) * s.nb + blockIdx.y;
        if (b >= s.B) return;
    } else if (blockIdx.y > 0) {
        return;
    }
    const int seq = s.seqs[b], r = threadIdx.x, key = m.z + r;
    if (seq < 0 || seq >= s.max_seqs) return;
    for (int j = 0; j < b; ++j)
        if (s.seqs[j] == seq) return;                  // listed before
    const int l = s.len[seq];
    if (key >= l || key >= m.w || l > s.max_pages * s.ps) return;
    float v = s.part[((size_t)blockIdx.x * s.nb + blockIdx.y) * KW_KEYS + r];
    for (int c = blockIdx.x / 2 + 1; c < s.G; ++c) {   // the unit goes on as the next CTAs' first piece
        v += s.part[((size_t)(2 * c) * s.nb + blockIdx.y) * KW_KEYS + r];
        if (s.meta[2 * c].x & KW_END) break;
    }
    float *at = s.w + (size_t)seq * s.w_ld + key;
    *at = s.decay == 0.0f ? v : fmaf(s.decay, *at, v);
}

// ------------------------------------------------------------ fp32 kernel
// 64 keys x 64 rows at a time, 256 threads as 16 x 16: thread (ty, tx) has rows 4 ty..
// and keys tx + 16 j.  A unit is 64 keys with all their rows, taken in turn.
constexpr int KF_KEYS = 64;
template <int HD>
__global__ void __launch_bounds__(256)
    key_weights_f32_kernel(const float *__restrict__ q, const long q_ld, const float *__restrict__ k,
                           const __grid_constant__ KeySched s, int *err) {
    constexpr int LD = HD + 4;
    extern __shared__ __align__(16) float sm[];
    __shared__ KeyLens L;
    __shared__ float sh_nl[64];
    __shared__ int sh_lim[64];
    float *sK = sm, *sQ = sm + 64 * LD;
    pdl_wait();
    pdl_release();
    key_lens<KF_KEYS>(s, L, err);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, log_ps = 31 - __clz(s.ps), rows = s.n_q * s.grp;
    const float scale = s.sl2;
    int b = 0, before = 0;                             // units of the branches before b
    for (int u = blockIdx.x;; u += gridDim.x) {
        while (b < s.B && u - before >= key_tiles<KF_KEYS>(s, L.len[b])) {
            before += key_tiles<KF_KEYS>(s, L.len[b]);
            ++b;
        }
        if (b == s.B) return;
        const int key0 = (u - before) * KF_KEYS, l = L.len[b], seq = L.seq[b];
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int h = 0; h < s.Hk; ++h) {
            __syncthreads();
            for (int x = tid; x < 64 * (HD / 4); x += 256) {
                const int r = x / (HD / 4), c = x - r * (HD / 4), key = key0 + r;
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (key < l) {
                    const int id = s.table[(size_t)seq * s.max_pages + (key >> log_ps)];
                    if (id >= 0 && id < s.n_pages)
                        v = reinterpret_cast<const float4 *>(k + ((size_t)id * s.ps + (key & (s.ps - 1))) * (s.Hk * HD) + h * HD)[c];
                    else if (err) atomicOr(err, ERR_BAD_SEQ);
                }
                *reinterpret_cast<float4 *>(sK + r * LD + 4 * c) = v;
            }
            const int i0 = s.causal ? max(key0 - (l - s.n_q), 0) : 0;      // the first token that sees the tile
            for (int r0 = i0 * s.grp; r0 < rows; r0 += 64) {
                __syncthreads();
                for (int x = tid; x < 64 * (HD / 4); x += 256) {
                    const int r = x / (HD / 4), c = x - r * (HD / 4);
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (r0 + r < rows) {
                        const int i = (r0 + r) / s.grp, g = r0 + r - i * s.grp;
                        v = reinterpret_cast<const float4 *>(q + (size_t)(b * s.n_q + i) * q_ld + (h * s.grp + g) * HD)[c];
                    }
                    *reinterpret_cast<float4 *>(sQ + r * LD + 4 * c) = v;
                }
                if (tid < 64) {
                    float nl = -INFINITY;
                    int lim = 0;
                    if (r0 + tid < rows) {
                        const int i = (r0 + tid) / s.grp, g = r0 + tid - i * s.grp;
                        nl = -s.lse[(size_t)(b * s.n_q + i) * (s.Hk * s.grp) + h * s.grp + g];
                        if (nl == INFINITY) nl = -INFINITY;
                        lim = s.limit(l, i) - key0;
                    }
                    sh_nl[tid] = nl;
                    sh_lim[tid] = lim;
                }
                __syncthreads();
                float a[4][4] = {};
#pragma unroll 4
                for (int d = 0; d < HD; d += 4) {
                    float4 qv[4], kv[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) qv[i] = *reinterpret_cast<const float4 *>(sQ + (4 * ty + i) * LD + d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4 *>(sK + (tx + 16 * j) * LD + d);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            a[i][j] = fmaf(qv[i].x, kv[j].x, a[i][j]);
                            a[i][j] = fmaf(qv[i].y, kv[j].y, a[i][j]);
                            a[i][j] = fmaf(qv[i].z, kv[j].z, a[i][j]);
                            a[i][j] = fmaf(qv[i].w, kv[j].w, a[i][j]);
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float nl = sh_nl[4 * ty + i];
                    const int lim = sh_lim[4 * ty + i];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (tx + 16 * j < lim) sum[j] += expf(fmaf(a[i][j], scale, nl));
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) sm[ty * 64 + tx + 16 * j] = sum[j];
        __syncthreads();
        if (tid < 64 && key0 + tid < l) {
            float v = 0.0f;
            for (int y = 0; y < 16; ++y) v += sm[y * 64 + tid];
            float *at = s.w + (size_t)seq * s.w_ld + key0 + tid;
            *at = s.decay == 0.0f ? v : fmaf(s.decay, *at, v);
        }
    }
}

// ------------------------------------------------------------------- host
static KeySched key_plan(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    KeySched s{};
    s.B = B;
    s.n_q = n_q;
    s.Hk = c.n_kv_heads;
    s.grp = H / s.Hk;
    s.max_seqs = c.max_seqs;
    s.max_pages = c.max_pages;
    s.ps = c.page_size;
    s.n_pages = c.n_pages;
    s.len = c.len;
    s.table = c.table;
    s.shared = shared;
    s.G = device_sms();
    s.nb = 1;
    s.tt = n_q;
    s.n_ct = 1;
    if (c.dtype == XC_F32) return s;
    // Branches' rows side by side, whole branches, where two or more fit a row tile.
    const long long tokens = (long long)B * n_q;
    s.packed = shared > 0 && B > 1 && 2ll * n_q * s.grp <= KW_COLS;
    s.tt = s.packed ? std::min(B, KW_COLS / (n_q * s.grp)) * n_q : std::min(KW_COLS / s.grp, n_q);
    s.N = (s.tt * s.grp + 15) / 16 * 16;
    s.n_ct = (int)(((s.packed ? tokens : n_q) + s.tt - 1) / s.tt);
    s.P = s.packed ? shared : 0;
    s.n_pt = (s.P + KW_KEYS - 1) / KW_KEYS;
    if (s.packed) s.nb = s.tt / n_q;
    return s;
}
bool key_weights_fit(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    const KeySched s = key_plan(c, B, n_q, H, shared);
    const long long tiles = ((long long)c.max_pages * c.page_size + KF_KEYS - 1) / KF_KEYS + 1;
    const long long ct = c.dtype == XC_F32 ? 1 : s.n_ct;
    return B <= KW_MAX_B && tiles * B * s.Hk * ct < (1ll << 31);
}
size_t key_weights_workspace_bytes(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    if (c.dtype == XC_F32) return 16;
    const KeySched s = key_plan(c, B, n_q, H, shared);
    return (size_t)2 * s.G * (sizeof(int4) + (size_t)s.nb * KW_KEYS * sizeof(float));
}

template <int HD, bool PACKED>
static cudaError_t key_launch_tc(const xc_kv_cache &c, const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    constexpr int K_BYTES = KW_KEYS * HD * 2, BUDGET = 200 * 1024;
    static bool done = false;
    if (!done) {
        const cudaError_t e = cudaFuncSetAttribute(key_weights_kernel<HD, PACKED>, cudaFuncAttributeMaxDynamicSharedMemorySize, BUDGET + 1024);
        if (e != cudaSuccess) return e;
        done = true;
    }
    const int q_bytes = s.N * HD * 2;
    KeyRing ring;
    ring.ks = s.n_ct > 2 && !PACKED ? 2 : std::min(8, BUDGET / (K_BYTES + q_bytes));
    ring.qs = std::min(8, (BUDGET - ring.ks * K_BYTES) / q_bytes);
    const uint64_t rows = (uint64_t)c.n_pages * c.page_size, cols = (uint64_t)c.n_kv_heads * HD;
    CUtensorMap tq, tk;
    if (!make_tmap_heads_bf16(&tq, a.q, HD, (uint64_t)s.Hk * s.grp, (uint64_t)s.B * s.n_q, a.q_ld, s.grp, s.tt) ||
        !make_tmap_bf16(&tk, a.k, rows, cols, c.page_size < KW_KEYS ? c.page_size : KW_KEYS))
        return cudaErrorInvalidValue;
    const cudaError_t e = launch_pdl(key_weights_kernel<HD, PACKED>, dim3(s.G), dim3(KW_THREADS),
                                     ring.ks * K_BYTES + ring.qs * q_bytes + 1024, st, tq, tk, s, ring, err);
    if (e != cudaSuccess) return e;
    return launch_pdl(key_merge_kernel, dim3(2 * s.G, s.nb), dim3(KW_KEYS), 0, st, s);
}
template <int HD>
static cudaError_t key_launch_f32(const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    constexpr int SMEM = 2 * 64 * (HD + 4) * 4;
    static bool done = false;
    if (!done && SMEM > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(key_weights_f32_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        if (e != cudaSuccess) return e;
    }
    done = true;
    return launch_pdl(key_weights_f32_kernel<HD>, dim3(4 * s.G), dim3(256), SMEM, st, reinterpret_cast<const float *>(a.q), a.q_ld,
                      reinterpret_cast<const float *>(a.k), s, err);
}

cudaError_t key_weights(const xc_kv_cache &c, const KeyWeightsArgs &a, void *ws, int *err, cudaStream_t st) {
    KeySched s = key_plan(c, a.B, a.n_q, a.H, a.shared);
    s.seqs = a.seqs;
    s.causal = a.causal;
    s.decay = a.decay;
    s.sl2 = c.dtype == XC_F32 ? a.scale : a.scale * KW_LOG2E;
    s.lse = a.lse;
    s.w = a.w;
    s.w_ld = a.w_ld;
    s.meta = reinterpret_cast<int4 *>(ws);
    s.part = reinterpret_cast<float *>(s.meta + 2 * s.G);
    if (c.dtype == XC_BF16) {
        if (c.head_dim == 64) return s.packed ? key_launch_tc<64, true>(c, a, s, err, st) : key_launch_tc<64, false>(c, a, s, err, st);
        if (c.head_dim == 128) return s.packed ? key_launch_tc<128, true>(c, a, s, err, st) : key_launch_tc<128, false>(c, a, s, err, st);
        return cudaErrorInvalidValue;
    }
    switch (c.head_dim) {
        case 16: return key_launch_f32<16>(a, s, err, st);
        case 32: return key_launch_f32<32>(a, s, err, st);
        case 64: return key_launch_f32<64>(a, s, err, st);
        case 128: return key_launch_f32<128>(a, s, err, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace xc
