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
// Four kernels.  Branches of few rows (single tokens, short chunks) wait for the keys'
// bytes, and where the branches share keys those are read once for the rows of as many branches as
// fit: key_weights_few_kernel takes few keys straight into registers (it begins sooner),
// key_weights_stream_kernel many through shared memory and tcgen05 products (it keeps more bytes under way).  Longer rows are
// products (key_weights_kernel, tcgen05) and exponentials; fp32 caches have a kernel of their own.
//
// What bf16 caches lose beside the exact sums comes from the scores: the tensor core drops the low bits of its partial
// sums (2^-23 of them, towards zero), which all rows share, so that sums over many do not average it out.  Scores of
// standard deviation 1, 2 and 4 at head size 128: 5e-8, 3.6e-7 and 1.4e-6 of a sum with tcgen05, 3e-8, 1.4e-7
// and 6e-7 with mma.sync; the exponentials, log2 units and fp32 additions make 6e-8 of it at 2.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "xc_branch.cuh"
#include "xc_ptx.cuh"

namespace xc {

constexpr int KW_MAX_B = 1024;           // branches of a call
constexpr int KW_TILE = 128, KW_KEYS = 2 * KW_TILE, KW_COLS = 128, KW_BUFS = 4;
constexpr int KW_SWAPS = 4;              // pieces of a step each that a column half may be ahead of the other, and more
constexpr float KW_LOG2E = 1.4426950408889634f;

struct KeySched {
    int B, n_q, grp, Hk, causal, G;
    int max_seqs, max_pages, ps, n_pages, shared;
    int P, n_pt;             // keys and key tiles of the shared units (few rows only; 0: none)
    int tt, N, n_ct;         // tokens and columns of a row tile; row tiles (of a branch; with shared units of all rows)
    int nb;                  // branches of a shared unit's row tile at most
    int wh, wk;              // few rows: warps over the key heads, over the keys
    int stream;              // few rows, many keys
    float decay, sl2;
    const int *seqs, *len, *table;
    const float *lse;        // [B n_q][Hk grp]
    float *w;
    long w_ld;
    int4 *meta;              // [2 G] what a CTA's cut pieces are
    float *part;             // [2 G][256]

    __device__ __forceinline__ int limit(int l, int i) const { return causal ? l - n_q + i + 1 : l; }
    __device__ __forceinline__ void put(int seq, int key, float v) const {
        float *at = w + (size_t)seq * w_ld + key;
        *at = decay == 0.0f ? v : fmaf(decay, *at, v);
    }
};
enum { KW_CUT = 1, KW_BEGIN = 2, KW_END = 4 };

// Lengths and sequences of the branches, and the line.  A sequence out of range, of an
// impossible length, or listed before has length 0 and takes no part.
struct KeyLens {
    int len[KW_MAX_B], seq[KW_MAX_B], off[KW_MAX_B + 1];
    int scan[32];
};

// Own tiles of kt keys of a branch of length l.
__device__ __forceinline__ int key_tiles(const KeySched &s, int l, int kt) { return l > s.P ? (l - s.P + kt - 1) / kt : 0; }
// Long rows: the first row tile that sees key tile t, and the steps of the tile.
__device__ __forceinline__ int key_first_ct(const KeySched &s, int l, int t) {
    if (!s.causal) return 0;
    const int i0 = t * KW_KEYS - (l - s.n_q);
    return i0 > 0 ? i0 / s.tt : 0;
}
__device__ __forceinline__ int key_steps(const KeySched &s, int l, int t) { return s.Hk * (s.n_ct - key_first_ct(s, l, t)); }
__device__ __forceinline__ int key_full_tiles(const KeySched &s, int l) {      // tiles that every row tile sees
    const int n = key_tiles(s, l, KW_KEYS);
    return !s.causal ? n : l < s.n_q ? 0 : min(n, (l - s.n_q) / KW_KEYS + 1);
}

// Every thread calls it.  Off: own units before each branch, of kt keys, or with STEPS
// the steps of the long rows' line.
template <bool STEPS>
__device__ void key_lens(const KeySched &s, KeyLens &L, int kt, int *err) {
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
        const int l = L.len[b];
        int x = key_tiles(s, l, kt);
        if constexpr (STEPS) {
            const int n = x, full = key_full_tiles(s, l);
            x = full * s.Hk * s.n_ct;
            for (int t = full; t < n; ++t) x += key_steps(s, l, t);
        }
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

// ------------------------------------------------------------------ long rows
// A unit is (branch, 256 keys), its steps the key heads x row tiles that see them.  All units'
// steps form one line that the CTAs share evenly, as in the attention: a unit that one CTA
// runs whole is written at once, the sums of a cut one leave as partials that key_merge_kernel
// adds in CTA order, so a call gives the same bits every time.
struct KeyPiece {
    int b, key0;             // branch, first key
    int t0, nct;             // first token of the first row tile; row tiles
    int s0, s1, n;           // steps of the piece, of the unit
};
struct KeyWalk {
    int b, t, off, left;
    __device__ __forceinline__ void start(const KeySched &s, const KeyLens &L, int c) {
        const unsigned T = L.off[s.B], q = T / s.G, r = T - q * s.G;
        const unsigned x = q * c + min((unsigned)c, r);
        left = q + ((unsigned)c < r ? 1 : 0);
        b = t = off = 0;
        if (left == 0) return;
        int lo = 0, hi = s.B;                          // the last b with off[b] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((unsigned)L.off[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo;
        int rest = x - L.off[b];
        const int l = L.len[b], each = s.Hk * s.n_ct, full = key_full_tiles(s, l);
        if (rest < full * each) {
            t = rest / each;
            off = rest - t * each;
            return;
        }
        rest -= full * each;
        for (t = full;; ++t) {
            const int n = key_steps(s, l, t);
            if (rest < n) break;
            rest -= n;
        }
        off = rest;
    }
    __device__ __forceinline__ bool next(const KeySched &s, const KeyLens &L, KeyPiece &p) {
        if (left <= 0) return false;
        while (t >= key_tiles(s, L.len[b], KW_KEYS)) {
            ++b;
            t = 0;
        }
        const int ct0 = key_first_ct(s, L.len[b], t);
        p.n = key_steps(s, L.len[b], t);
        p.b = b;
        p.key0 = t * KW_KEYS;
        p.t0 = b * s.n_q + ct0 * s.tt;
        p.nct = s.n_ct - ct0;
        p.s0 = off;
        p.s1 = min(p.n, off + left);
        left -= p.s1 - p.s0;
        off = 0;
        ++t;
        return true;
    }
};

// Warps: 0 loads (two key tiles of 128 page by page, row tiles), 1 issues the products, 2 reads
// the rows' lse and limits, 4-19 take the exponentials: eight for either key tile, thread = key,
// two warps per TMEM quadrant, half of the columns each.  Two key tiles, as every row tile is read from
// L2 for both: with one, the rows came too late for the products (2 x 4320 queries over 30240 keys, 12 heads x 128:
// 932 us, with two 735).  Products and exponentials take 1024 cycles each of a step's 2200; the tensor pipe, the
// special-function unit and the issue slots are at 48 % each: the softmax warps' wait, load and exponentials
// follow one another.  All sixteen warps on every tile: 1040 us.  A share of the exponentials on the FMA pipe (Cody and
// Waite's reduction and a polynomial) was slower still.
constexpr int KW_SOFT = 512, KW_THREADS = 128 + KW_SOFT;
struct alignas(16) KeyCols { // what a step's columns need
    float nl[KW_COLS];       // -lse log2(e)
    int lim[KW_COLS];        // keys of the unit that the column's row sees
    int masked;
};

// Four products of a step, S^T (+)= K Q^T over 64 numbers of the head, by one elected lane.
__device__ __forceinline__ void key_issue4(uint32_t acc, uint64_t k, uint64_t q, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred e, p, t;\n\t.reg .b32 r;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "elect.sync r|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.eq.b32 t, %4, %4;\n\t"
        "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, t;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, t;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, t;\n\t}"
        ::"r"(acc), "l"(k), "l"(q), "r"(idesc), "r"(add)
        : "memory");
}

template <int HD>
__global__ void __launch_bounds__(KW_THREADS, 1)
    key_weights_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ KeySched s, const int q_slots, int *err) {
    constexpr int NR = HD / 64, K_REGION = KW_TILE * 128, K_BYTES = NR * K_REGION;
    extern __shared__ uint8_t smem_raw[];
    __shared__ KeyLens L;
    __shared__ KeyCols cols[KW_BUFS / 2];
    __shared__ float sh_sum[KW_SWAPS][KW_KEYS];
    __shared__ uint64_t bars[4 + 16 + 2 * KW_BUFS + KW_SWAPS + 1];
    __shared__ uint32_t tmem_slot;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int q_region = s.N * 128, q_bytes = NR * q_region;
    uint8_t *sK = smem, *sQ = smem + 2 * K_BYTES;
    uint64_t *k_full = bars, *k_empty = bars + 2, *q_full = bars + 4, *q_empty = bars + 12;     // [2] key tiles, [8] row tiles
    uint64_t *s_full = bars + 20, *s_empty = s_full + KW_BUFS;          // s_full: the scores and the columns' lse
    uint64_t *swap = s_empty + KW_BUFS, *drained = swap + KW_SWAPS;     // swap: the second half's sums are in sh_sum
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1);
        }
        for (int i = 0; i < 8; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < KW_BUFS; ++i) {
            mbar_init(&s_full[i], 33);
            mbar_init(&s_empty[i], KW_SOFT / 2);
        }
        for (int i = 0; i < KW_SWAPS; ++i) mbar_init(&swap[i], KW_SOFT / 2);
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(&tmem_slot, 512);
    // columns that no row tile fills stay zero
    for (int x = threadIdx.x; x < q_slots * q_bytes / 16; x += KW_THREADS) reinterpret_cast<uint4 *>(sQ)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    pdl_wait();
    key_lens<true>(s, L, KW_KEYS, err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = 0;                           // all 512 columns are this CTA's
    KeyWalk walk;
    walk.start(s, L, blockIdx.x);
    KeyPiece p;

    if (warp == 0) {
        const int box = min(s.ps, KW_TILE), log_ps = 31 - __clz(s.ps);
        int qi = 0, kc = 0, qc = 0;
        uint32_t q_ph = 1, k_ph = 1;
        bool ok = true;
        while (ok && walk.next(s, L, p)) {
            const int seq = L.seq[p.b];
            int row[2];                                // first pool row of this lane's page of either tile
            uint32_t k_tx[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = p.key0 + t * KW_TILE + lane * box;
                row[t] = -1;
                if (lane * box < KW_TILE && key < L.len[p.b]) {
                    const int id = s.table[(size_t)seq * s.max_pages + (key >> log_ps)];
                    const bool good = id >= 0 && id < s.n_pages;
                    if (!good && err) atomicOr(err, ERR_BAD_SEQ);
                    row[t] = good ? id * s.ps + (key & (s.ps - 1)) : s.n_pages * s.ps;      // out of range: TMA fills zeros
                }
                k_tx[t] = __popc(__ballot_sync(0xffffffffu, row[t] >= 0)) * box * 128 * NR;
            }
            int h = p.s0 / p.nct, ct = p.s0 - h * p.nct;
            for (int st = p.s0; st < p.s1; ++st, ++qc) {
                if (st == p.s0 || ct == 0) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        ok = ok && mbar_wait(&k_empty[t], k_ph, err, ERR_WAIT_PRODUCER);
                        if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                        if (lane == 0) mbar_expect_tx(&k_full[t], k_tx[t]);
                        __syncwarp();
                        if (row[t] >= 0)
                            for (int r = 0; r < NR; ++r)
                                tma_load_2d(sK + t * K_BYTES + r * K_REGION + lane * box * 128, &tmK, &k_full[t], h * HD + 64 * r, row[t]);
                    }
                    if (!ok) break;
                    k_ph ^= 1;
                    ++kc;
                }
                ok = mbar_wait(&q_empty[qi], q_ph, err, ERR_WAIT_PRODUCER);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                if (lane == 0) {
                    mbar_expect_tx(&q_full[qi], NR * s.tt * s.grp * 128);
                    for (int r = 0; r < NR; ++r)
                        tma_load_3d(sQ + qi * q_bytes + r * q_region, &tmQ, &q_full[qi], 64 * r, h * s.grp, p.t0 + ct * s.tt);
                }
                __syncwarp();
                if (++qi == q_slots) {
                    qi = 0;
                    q_ph ^= 1;
                }
                if (++ct == p.nct) {
                    ct = 0;
                    ++h;
                }
            }
        }
        if (lane == 0) {                               // every copy has landed before the CTA exits
            for (int t = 0; t < 2 && kc > 0; ++t) mbar_wait(&k_full[t], (kc - 1) & 1, err, ERR_WAIT_PRODUCER);
            for (int j = max(qc - q_slots, 0); j < qc; ++j) mbar_wait(&q_full[j % q_slots], (j / q_slots) & 1, err, ERR_WAIT_PRODUCER);
        }
    } else if (warp == 1) {
        const uint32_t idesc = idesc_bf16(KW_TILE, 16, false, false) - ((16u >> 3) << 17) + ((uint32_t)(s.N >> 3) << 17);
        const uint64_t dK = sdesc_sw128(smem_u32(sK), 16, 1024), dQ = sdesc_sw128(smem_u32(sQ), 16, 1024);
        auto wait = [&](uint64_t *b, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(b, parity & 1, err, ERR_WAIT_MMA)) != 0;
        };
        int qi = 0, buf = 0;
        uint32_t k_ph = 0, q_ph = 0, s_ph = 1;
        bool ok = true, there[2] = {false, false};     // the next step's rows and buffers have been seen to be ready
        while (ok && walk.next(s, L, p)) {
            int ct = p.s0 % p.nct;
            for (int st = p.s0; ok && st < p.s1; ++st) {
                const bool first = st == p.s0 || ct == 0, last = ct + 1 == p.nct || st + 1 == p.s1;      // of the key tiles
                const uint64_t db = dQ + (uint64_t)((qi * q_bytes) >> 4);
                uint64_t *q_done = &q_empty[qi];
                const int buf0 = buf, q_next = qi + 1 == q_slots ? 0 : qi + 1;
                const uint32_t s_ph0 = s_ph, q_ph0 = q_ph, q_ph_next = q_next == 0 ? q_ph ^ 1 : q_ph;
                const int qi0 = qi;
                buf = buf == KW_BUFS - 2 ? 0 : buf + 2;
                s_ph ^= buf == 0 ? 1 : 0;
                const bool t0 = there[0], t1 = there[1];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (first && !(ok = wait(&k_full[t], k_ph))) break;
                    if (!__all_sync(0xffffffffu, t == 0 ? t0 : t1) &&
                        !(ok = (t == 1 || wait(&q_full[qi0], q_ph0)) && wait(&s_empty[buf0 + t], s_ph0))) break;
                    tc_fence_after();
                    there[t] = mbar_test2(&q_full[q_next], q_ph_next, &s_empty[buf + t], s_ph);
                    const uint64_t da = dK + (uint64_t)((t * K_BYTES) >> 4);
#pragma unroll
                    for (int r = 0; r < NR; ++r)
                        key_issue4(tmem + (buf0 + t) * KW_COLS, da + (uint64_t)((r * K_REGION) >> 4), db + (uint64_t)((r * q_region) >> 4), idesc, r);
                    if (last) tc_commit_warp(&k_empty[t]);
                    if (t == 1) tc_commit_warp(q_done);
                    tc_commit_warp(&s_full[buf0 + t]);
                }
                if (first) k_ph ^= 1;
                if (++ct == p.nct) ct = 0;
                qi = q_next;
                q_ph = q_ph_next;
            }
        }
        if (!ok) {                                     // a wait ran out: no product is under way when the CTA ends
            tc_commit_warp(drained);
            wait(drained, 0);
        }
    } else if (warp == 2) {
        // lse and limits of a step's columns, read a step ahead of when they are stored
        int tk[4], gq[4], it = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 32 * i;
            tk[i] = c / s.grp;
            gq[i] = c - tk[i] * s.grp;
        }
        float nl[4];
        int lim[4];
        bool masked = false;
        auto read = [&](const KeyPiece &x, int st) {
            const int h = st / x.nct, t0 = x.t0 + (st - h * x.nct) * s.tt, t_end = (x.b + 1) * s.n_q, l = L.len[x.b];
            masked = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + tk[i];
                nl[i] = -INFINITY;
                lim[i] = 0;
                if (lane + 32 * i < s.N) {
                    if (tk[i] < s.tt && t < t_end) {
                        nl[i] = s.lse[(size_t)t * (s.Hk * s.grp) + h * s.grp + gq[i]];
                        lim[i] = min(max(s.limit(l, t - x.b * s.n_q) - x.key0, 0), KW_KEYS);
                    }
                    masked = masked || lim[i] < KW_KEYS;
                }
            }
        };
        bool ok = true, more = walk.next(s, L, p);
        int st = p.s0;
        if (more) read(p, st);
        while (ok && more) {
            const int b2 = it & 1;
            const uint32_t ph = ((it >> 1) & 1) ^ 1;
            float v[4];
            int m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {              // a row that saw no key adds nothing
                v[i] = nl[i] == -INFINITY ? -INFINITY : -KW_LOG2E * nl[i];
                m[i] = lim[i];
            }
            const bool any = __any_sync(0xffffffffu, masked) != 0;
            if (++st >= p.s1) {
                more = walk.next(s, L, p);
                st = p.s0;
            }
            if (more) read(p, st);
            ok = mbar_wait(&s_empty[2 * b2], ph, err, ERR_WAIT_SOFTMAX) && mbar_wait(&s_empty[2 * b2 + 1], ph, err, ERR_WAIT_SOFTMAX);
            if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cols[b2].nl[lane + 32 * i] = v[i];
                cols[b2].lim[lane + 32 * i] = m[i];
            }
            if (lane == 0) cols[b2].masked = any;
            mbar_arrive(&s_full[2 * b2]);
            mbar_arrive(&s_full[2 * b2 + 1]);
            ++it;
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = ((warp - 4) >> 2) & 1, tile = (warp - 4) >> 3, r = tile * KW_TILE + 32 * q + lane;   // key of the unit
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16) + tile * KW_COLS;
        // this thread's columns, by 16: four of 8, or fewer
        const int nc = s.N / 16, ch0 = half * ((nc + 1) / 2), n_ch = half ? nc / 2 : (nc + 1) / 2, c0 = 16 * ch0;
        const float2 sl2 = make_float2(s.sl2, s.sl2);
        if (warp == 4 && lane < 2) s.meta[2 * blockIdx.x + lane] = make_int4(0, 0, 0, 0);
        __syncwarp();
        int it = 0, np = 0;
        bool ok = true;
        while (ok && walk.next(s, L, p)) {
            float acc = 0.0f;
            for (int st = p.s0; st < p.s1; ++st, ++it) {
                const int b2 = it & 1;
                ok = mbar_wait(&s_full[2 * b2 + tile], (it >> 1) & 1, err, ERR_WAIT_SOFTMAX);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                tc_fence_after();
                const KeyCols &kc = cols[b2];
                const uint32_t at = lanes + 2 * b2 * KW_COLS + c0;
                float2 sum0 = make_float2(0.0f, 0.0f), sum1 = sum0;
                // exponentials of n columns from column c
                auto run = [&](auto n_, auto masked_, int c, const float *x) {
                    constexpr int n = decltype(n_)::value;
                    constexpr bool masked = decltype(masked_)::value;
#pragma unroll
                    for (int i = 0; i < n; i += 4) {
                        const float4 nl = *reinterpret_cast<const float4 *>(&kc.nl[c + i]);
                        float2 a = __ffma2_rn(make_float2(x[i], x[i + 1]), sl2, make_float2(nl.x, nl.y));
                        float2 b = __ffma2_rn(make_float2(x[i + 2], x[i + 3]), sl2, make_float2(nl.z, nl.w));
                        a = make_float2(exp2_mufu(a.x), exp2_mufu(a.y));
                        b = make_float2(exp2_mufu(b.x), exp2_mufu(b.y));
                        if constexpr (masked) {
                            const int4 lim = *reinterpret_cast<const int4 *>(&kc.lim[c + i]);
                            a = make_float2(r < lim.x ? a.x : 0.0f, r < lim.y ? a.y : 0.0f);
                            b = make_float2(r < lim.z ? b.x : 0.0f, r < lim.w ? b.y : 0.0f);
                        }
                        sum0 = __fadd2_rn(sum0, a);
                        sum1 = __fadd2_rn(sum1, b);
                    }
                };
                if (n_ch == 4) {
                    float x[64];
                    tmem_ld64_sync(at, x);
                    if (kc.masked) run(std::integral_constant<int, 64>(), std::true_type(), c0, x);
                    else run(std::integral_constant<int, 64>(), std::false_type(), c0, x);
                } else {
                    for (int k = 0; k < n_ch; ++k) {
                        float x[16];
                        tmem_ld16_sync(at + 16 * k, x);
                        run(std::integral_constant<int, 16>(), std::true_type(), c0 + 16 * k, x);
                    }
                }
                sum0 = __fadd2_rn(sum0, sum1);
                acc += sum0.x + sum0.y;
                tc_fence_before();
                mbar_arrive(&s_empty[2 * b2 + tile]);
            }
            if (!ok) break;
            const bool whole = p.s1 - p.s0 == p.n;
            const int slot = 2 * blockIdx.x + (np == 0 ? 0 : 1), key = p.key0 + r, sw = np % KW_SWAPS;
            if (!whole && warp == 4 && lane == 0)
                s.meta[slot] = make_int4(KW_CUT | (p.s0 == 0 ? KW_BEGIN : 0) | (p.s1 == p.n ? KW_END : 0), p.b, p.key0, 0);
            if (half == 1) {
                sh_sum[sw][r] = acc;
                mbar_arrive(&swap[sw]);
            } else {
                ok = __all_sync(0xffffffffu, mbar_wait(&swap[sw], (np / KW_SWAPS) & 1, err, ERR_WAIT_SOFTMAX)) != 0;
                if (!ok) break;
                acc += sh_sum[sw][r];
                if (!whole) s.part[(size_t)slot * KW_KEYS + r] = acc;
                else if (key < L.len[p.b]) s.put(L.seq[p.b], key, acc);
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

// Adds the pieces of a cut unit in CTA order.
__global__ void __launch_bounds__(KW_KEYS) key_merge_kernel(const __grid_constant__ KeySched s) {
    pdl_wait();
    pdl_release();
    const int4 m = s.meta[blockIdx.x];
    if ((m.x & KW_CUT) == 0 || (m.x & KW_BEGIN) == 0) return;
    const int seq = s.seqs[m.y], r = threadIdx.x, key = m.z + r;
    if (key >= s.len[seq]) return;
    float v = s.part[(size_t)blockIdx.x * KW_KEYS + r];
    for (int c = blockIdx.x / 2 + 1; c < s.G; ++c) {   // the unit goes on as the next CTAs' first piece
        v += s.part[(size_t)(2 * c) * KW_KEYS + r];
        if (s.meta[2 * c].x & KW_END) break;
    }
    s.put(seq, key, v);
}

// ------------------------------------------------------------------- few rows
// A unit is 16 wk keys with the rows of one branch, or (shared keys) of as many branches as fit
// 64 columns.  A warp takes 16 of the keys and every wh-th key head: it loads the keys
// straight into the registers of the MMA's A operand (16 consecutive numbers of a lane are its part of two
// products; the rows, in shared memory, are laid out to match), the next head's or unit's while it
// computes, and keeps a sum for every column.  The warps' sums meet in shared memory at the
// unit's end (two places in turn, so that one barrier a unit is enough), in a fixed order, and one thread
// writes each (branch, key), whose old weight it read when the unit began.  Latency bounds it: 4 single tokens,
// 8 heads x 64, 2016 keys 6.7 us.
constexpr int KFEW_THREADS = 512, KFEW_WARPS = KFEW_THREADS / 32, KFEW_COLS = 64, KFEW_PITCH = 20;
constexpr size_t KFEW_SMEM = 208 * 1024;

__device__ __forceinline__ void mma_bf16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Unit u: its branch (own) or row tile (shared), and its first key.
struct KeyUnit {
    int own, b, key0, end;   // end: behind the last key
    __device__ __forceinline__ KeyUnit(const KeySched &s, const KeyLens &L, int u, int kt) {
        const int shared = s.n_pt * s.n_ct;
        own = u >= shared;
        if (!own) {
            b = u / s.n_pt;
            key0 = (u - b * s.n_pt) * kt;
            end = s.P;
            return;
        }
        const int x = u - shared;
        int lo = 0, hi = s.B;                          // the last b with off[b] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (L.off[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo;
        key0 = s.P + (x - L.off[b]) * kt;
        end = L.len[b];
    }
};

template <int HD, int NT>
__global__ void __launch_bounds__(KFEW_THREADS, 1)
    key_weights_few_kernel(const bf16 *__restrict__ q, const long q_ld, const bf16 *__restrict__ k, const __grid_constant__ KeySched s, int *err) {
    constexpr int CH = HD / 32;                        // 16-byte parts of a lane's key row
    extern __shared__ __align__(16) uint4 sm_few[];
    __shared__ KeyLens L;
    __shared__ __align__(8) int sh_lim[KFEW_COLS];
    __shared__ int sh_least;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    constexpr int ncol = 8 * NT;
    const int log_kt = 4 + 31 - __clz(s.wk), kt = 1 << log_kt, wh = warp % s.wh, wk = warp / s.wh;
    uint4 *sQ = sm_few;                                // [Hk][CH][ncol][4]
    float *sNl = reinterpret_cast<float *>(sQ + (size_t)s.Hk * CH * ncol * 4);     // [Hk][ncol]
    float *red = sNl + s.Hk * ncol;                    // [2][warps][ncol][KFEW_PITCH]
    pdl_wait();
    key_lens<false>(s, L, kt, err);
    pdl_release();
    const int log_ps = 31 - __clz(s.ps);
    const int U = s.n_pt * s.n_ct + L.off[s.B], u0 = (int)((long long)U * blockIdx.x / gridDim.x), u1 = (int)((long long)U * (blockIdx.x + 1) / gridDim.x);
    if (u0 == u1) return;
    // Table entry of this warp's 16 keys of unit u (loaded, not looked at), and the first one's place in the page;
    // the pool row that it makes, -1: no keys, -2: a bad page.
    auto entry = [&](int u, int &id, int &at) {
        id = 0;
        at = -1;
        if (u >= u1) return;
        const KeyUnit x(s, L, u, kt);
        const int key = x.key0 + 16 * wk, seq = L.seq[x.own ? x.b : 0];
        if (key >= x.end) return;
        at = key & (s.ps - 1);
        id = seq >= 0 && seq < s.max_seqs ? s.table[(size_t)seq * s.max_pages + (key >> log_ps)] : -1;
    };
    auto pool_row = [&](int id, int at) -> long {
        if (at < 0) return -1;
        if (id < 0 || id >= s.n_pages) {
            if (err) atomicOr(err, ERR_BAD_SEQ);
            return -2;
        }
        return (long)id * s.ps + at;
    };
    auto load = [&](long row, int h, uint4 (&x)[2][CH]) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int c = 0; c < CH; ++c)
                x[r][c] = row >= 0 ? *reinterpret_cast<const uint4 *>(k + ((size_t)(row + gid + 8 * r) * s.Hk + h) * HD + 32 * c + 8 * tig)
                                   : make_uint4(0, 0, 0, 0);
    };
    int id0, at0, id1, at1;
    entry(u0, id0, at0);
    entry(u0 + 1, id1, at1);
    long row = pool_row(id0, at0), row_next = pool_row(id1, at1);
    uint4 x[2][CH];
    if (wh < s.Hk) load(row, wh, x);
    int have_own = -1, have_b = -1;                    // whose rows are in shared memory
    for (int u = u0; u < u1; ++u) {
        const KeyUnit unit(s, L, u, kt);
        const int t0 = unit.own ? unit.b * s.n_q : unit.b * s.tt;
        const int tokens = unit.own ? s.n_q : min(s.tt, s.B * s.n_q - t0), cols = tokens * s.grp;
        if (unit.own != have_own || unit.b != have_b) {
            have_own = unit.own;
            have_b = unit.b;
            __syncthreads();                           // the last unit's rows have been used
            const int parts = s.Hk * ncol * CH * 4;
            constexpr int BATCH = 6;                   // loads in flight
            for (int y0 = tid; y0 < parts; y0 += BATCH * KFEW_THREADS) {
                uint4 v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int y = y0 + i * KFEW_THREADS, part = y % (CH * 4), rest = y / (CH * 4), c = rest % ncol, h = rest / ncol;
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (y < parts && c < cols)
                        v[i] = *reinterpret_cast<const uint4 *>(q + (size_t)(t0 + c / s.grp) * q_ld + (h * s.grp + c % s.grp) * HD + 8 * part);
                }
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int y = y0 + i * KFEW_THREADS, part = y % (CH * 4), rest = y / (CH * 4), c = rest % ncol, h = rest / ncol;
                    if (y < parts) sQ[((h * CH + part / 4) * ncol + c) * 4 + part % 4] = v[i];
                }
            }
            for (int y = tid; y < s.Hk * ncol; y += KFEW_THREADS) {
                const int c = y % ncol, h = y / ncol;
                float v = -INFINITY;
                if (c < cols) v = s.lse[(size_t)(t0 + c / s.grp) * (s.Hk * s.grp) + h * s.grp + c % s.grp];
                sNl[y] = v == -INFINITY ? -INFINITY : -KW_LOG2E * v;       // a row that saw no key adds nothing
            }
            if (tid == 0) sh_least = INT_MAX;
            __syncthreads();
            if (tid < ncol) {
                int lim = 0;
                if (tid < cols) {
                    const int t = t0 + tid / s.grp, b = t / s.n_q;
                    lim = s.limit(L.len[b], t - b * s.n_q);
                    atomicMin(&sh_least, lim);
                }
                sh_lim[tid] = lim;
            }
            __syncthreads();
        }
        entry(u + 2, id1, at1);                        // the table's entry comes while this unit is computed
        const int key = unit.key0 + 16 * wk;           // this warp's first key
        const bool masked = key + 16 > sh_least, there = key < unit.end;
        // this thread's outputs, (branch j, key r) of the unit: the first two
        const int each = s.n_q * s.grp, outs = (unit.own ? 1 : tokens / s.n_q) * kt;
        float *at_w[2];
        float old[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int y = tid + i * KFEW_THREADS, j = y >> log_kt, r = y & (kt - 1), ky = unit.key0 + r;
            at_w[i] = nullptr;
            if (y < outs) {
                const int b = unit.own ? unit.b : unit.b * s.nb + j;
                if (ky < unit.end && ky < L.len[b]) at_w[i] = s.w + (size_t)L.seq[b] * s.w_ld + ky;
            }
            old[i] = at_w[i] != nullptr && s.decay != 0.0f ? *at_w[i] : 0.0f;
        }
        float acc[NT][4] = {};
        for (int h = wh; h < s.Hk; h += s.wh) {
            uint4 a[2][CH];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < CH; ++c) a[r][c] = x[r][c];
            const bool same = h + s.wh < s.Hk;
            load(same ? row : row_next, same ? h + s.wh : wh, x);
            if (!there) continue;
            const uint4 *qh = sQ + (size_t)h * CH * ncol * 4 + 4 * gid + tig;
            const float *nl = sNl + h * ncol + 2 * tig;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float sc[2][4] = {};
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const uint4 b = qh[(c * ncol + 8 * n) * 4];
                    mma_bf16(sc[0], a[0][c].x, a[1][c].x, a[0][c].y, a[1][c].y, b.x, b.y);
                    mma_bf16(sc[1], a[0][c].z, a[1][c].z, a[0][c].w, a[1][c].w, b.z, b.w);
                }
                const float2 l = *reinterpret_cast<const float2 *>(nl + 8 * n);
                float p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = exp2_mufu(fmaf(sc[0][j] + sc[1][j], s.sl2, j & 1 ? l.y : l.x));
                if (masked) {
                    const int2 lim = *reinterpret_cast<const int2 *>(&sh_lim[8 * n + 2 * tig]);
                    if (key + gid >= lim.x) p[0] = 0.0f;
                    if (key + gid >= lim.y) p[1] = 0.0f;
                    if (key + gid + 8 >= lim.x) p[2] = 0.0f;
                    if (key + gid + 8 >= lim.y) p[3] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[n][j] += p[j];
            }
        }
        float *place = red + (u & 1) * KFEW_WARPS * ncol * KFEW_PITCH, *mine = place + warp * ncol * KFEW_PITCH;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float *at = mine + (8 * n + 2 * tig) * KFEW_PITCH + gid;
            at[0] = acc[n][0];
            at[KFEW_PITCH] = acc[n][1];
            at[8] = acc[n][2];
            at[KFEW_PITCH + 8] = acc[n][3];
        }
        __syncthreads();
        // the warps of the key's 16, the branch's columns; a warp writes the next unit's sums elsewhere, and those
        // after them behind a barrier that this comes before
        auto total = [&](int y) {
            const int j = y >> log_kt, r = y & (kt - 1);
            const float *at = place + ((r >> 4) * s.wh * ncol + j * each) * KFEW_PITCH + (r & 15);
            float v0 = 0.0f, v1 = 0.0f, v2 = 0.0f, v3 = 0.0f;
            for (int w = 0; w < s.wh; ++w, at += ncol * KFEW_PITCH) {
                const float *p = at;
                int c = each;
#pragma unroll 2
                for (; c >= 4; c -= 4, p += 4 * KFEW_PITCH) {
                    v0 += p[0];
                    v1 += p[KFEW_PITCH];
                    v2 += p[2 * KFEW_PITCH];
                    v3 += p[3 * KFEW_PITCH];
                }
                if (c > 0) v0 += p[0];
                if (c > 1) v1 += p[KFEW_PITCH];
                if (c > 2) v2 += p[2 * KFEW_PITCH];
            }
            return (v0 + v1) + (v2 + v3);
        };
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (at_w[i] != nullptr) {
                const float sum = total(tid + i * KFEW_THREADS);
                *at_w[i] = s.decay == 0.0f ? sum : fmaf(s.decay, old[i], sum);
            }
        for (int y = tid + 2 * KFEW_THREADS; y < outs; y += KFEW_THREADS) {      // many branches of one key head
            const int j = y >> log_kt, ky = unit.key0 + (y & (kt - 1)), b = unit.own ? unit.b : unit.b * s.nb + j;
            if (ky < unit.end && ky < L.len[b]) s.put(L.seq[b], ky, total(y));
        }
        row = row_next;
        row_next = pool_row(id1, at1);
    }
}

// ---------------------------------------------------------- few rows, many keys
// A tile is 128 keys with the rows of one branch, or (shared keys) of as many branches as fit 64
// columns; the CTAs share the line of all tiles evenly (shares in finer steps have more tiles, which
// cost more than their keys: 4 single tokens over 16384 keys of 12 heads x 128 took 20 us instead of 15).  A step is
// a tile and a key head: its keys and rows come by TMA, several steps ahead, so that the
// keys' bytes bound it.  Warps: 0 loads, 1 issues the products, 2 reads the rows' lse and limits, two groups
// of four take the exponentials of every other step; thread = key, which adds up each branch's columns in shared
// memory of its own over the key heads, and the groups in turn write a tile's weights.  Up to eight columns a
// branch are added up by code for just that many: with a test at each column a step of 48 took 1.75 us.
// 8 single tokens, 40 / 8 heads x 128, 38880 shared + 1..1500 own keys: 25.8 us (in registers 49.4), 7 until the first
// tile is there, then 6.3 TB/s.  At most KST_NB branches a tile: with 8, 16 and 32, 32 branches over 8192 shared keys of
// 12 heads x 128 took 21.4, 24.3 and 21.3 us, over 32768 keys 64.6, 46.1 and 40.3, 64 over 16384 of 8 x 64
// 43.4, 38.5 and 41.3: fewer tiles read the keys less often, more have smaller sums and more slots.
constexpr int KST_SOFT = 256, KST_THREADS = 128 + KST_SOFT, KST_COLS = 64, KST_BUFS = 8, KST_SLOTS = 8, KST_NB = 16, KST_BUDGET = 204 * 1024;
// Key bytes, with every table row full, from which few rows go as a stream: below, its barriers and first copies take
// longer than the keys (4 single tokens, 8 heads x 64: 4096 keys 9.6 us against 6.7, 16384 keys 10.9 against
// 13.7; 12 heads x 128: 4096 keys 12.2 against 10.9, 8192 keys 12.8 against 15.9).  The host has the tables' width
// and not the lengths, so short sequences in wide tables pay that: 2016 keys a branch of 8 x 64 in rows of
// 2048 8.5 us, of 4096 9.2 (two caches in turn).
constexpr long long KST_BYTES = 12 << 20;

struct KeyRun {
    int own, b, key0, end;               // end: behind the last key
    int t0, tokens;                      // its rows
};
struct KeyRuns {
    int u, u1;
    __device__ __forceinline__ KeyRuns(const KeySched &s, const KeyLens &L) {
        const long long U = s.n_pt * s.n_ct + L.off[s.B];
        u = (int)(U * blockIdx.x / gridDim.x);
        u1 = (int)(U * (blockIdx.x + 1) / gridDim.x);
    }
    __device__ __forceinline__ bool next(const KeySched &s, const KeyLens &L, KeyRun &r) {
        if (u >= u1) return false;
        const KeyUnit x(s, L, u++, KW_TILE);
        r.own = x.own;
        r.b = x.b;
        r.key0 = x.key0;
        r.end = min(x.end, x.key0 + KW_TILE);
        r.t0 = x.own ? x.b * s.n_q : x.b * s.tt;
        r.tokens = x.own ? s.n_q : min(s.tt, s.B * s.n_q - r.t0);
        return true;
    }
};

template <int HD>
__global__ void __launch_bounds__(KST_THREADS, 1)
    key_weights_stream_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                              const __grid_constant__ KeySched s, const int slots, int *err) {
    constexpr int NR = HD / 64, K_REGION = KW_TILE * 128, K_BYTES = NR * K_REGION;
    extern __shared__ uint8_t smem_raw[];
    __shared__ KeyLens L;
    __shared__ KeyCols cols[KST_BUFS];
    __shared__ uint64_t bars[2 * KST_SLOTS + 2 * KST_BUFS + 5];
    __shared__ uint32_t tmem_slot;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int q_region = s.N * 128, slot_bytes = K_BYTES + NR * q_region;
    float *sums = reinterpret_cast<float *>(smem + slots * slot_bytes);            // [2 tiles in turn][2 groups][nb][128]
    uint64_t *full = bars, *empty = bars + KST_SLOTS, *s_full = empty + KST_SLOTS, *s_empty = s_full + KST_BUFS;
    uint64_t *added = s_empty + KST_BUFS, *taken = added + 2, *drained = taken + 2;         // a tile's sums are complete; have been read
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < KST_BUFS; ++i) {
            mbar_init(&s_full[i], 33);
            mbar_init(&s_empty[i], KST_SOFT / 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&added[i], KST_SOFT);
            mbar_init(&taken[i], KST_SOFT / 2);
        }
        mbar_init(drained, 1);
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(&tmem_slot, 512);
    for (int i = 0; i < slots; ++i)                    // columns that no rows fill stay zero
        for (int x = threadIdx.x; x < NR * q_region / 16; x += KST_THREADS)
            reinterpret_cast<uint4 *>(smem + i * slot_bytes + K_BYTES)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    pdl_wait();
    key_lens<false>(s, L, KW_TILE, err);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = 0;                           // all 512 columns are this CTA's
    KeyRuns runs(s, L);
    KeyRun r;

    if (warp == 0) {
        const int log_ps = 31 - __clz(s.ps), box = min(s.ps, KW_TILE);
        auto boxes = [&](const KeyRun &x) { return (x.end - x.key0 + box - 1) / box; };
        auto entry = [&](const KeyRun &x) {            // table entry of this lane's keys
            const int seq = L.seq[x.own ? x.b : 0];
            if (lane >= boxes(x) || seq < 0 || seq >= s.max_seqs) return -1;
            return s.table[(size_t)seq * s.max_pages + ((x.key0 + lane * box) >> log_ps)];
        };
        int i = 0, it = 0;
        uint32_t ph = 1;
        bool ok = true, more = runs.next(s, L, r);
        int id = more ? entry(r) : -1;
        while (ok && more) {
            int row = s.n_pages * s.ps;                // out of range: TMA fills zeros
            const int n = boxes(r), t0 = r.t0, tx = NR * 128 * (n * box + s.tt * s.grp);
            if (lane < n) {
                if (id >= 0 && id < s.n_pages) row = id * s.ps + ((r.key0 + lane * box) & (s.ps - 1));
                else if (err) atomicOr(err, ERR_BAD_SEQ);
            }
            more = runs.next(s, L, r);
            id = more ? entry(r) : -1;                 // on its way while this tile is loaded
            for (int h = 0; h < s.Hk; ++h, ++it) {
                ok = mbar_wait(&empty[i], ph, err, ERR_WAIT_PRODUCER);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                uint8_t *slot = smem + i * slot_bytes;
                if (lane == 0) {
                    mbar_expect_tx(&full[i], tx);
                    for (int k = 0; k < NR; ++k)
                        tma_load_3d(slot + K_BYTES + k * q_region, &tmQ, &full[i], 64 * k, h * s.grp, t0);
                }
                __syncwarp();
                if (lane < n)
                    for (int k = 0; k < NR; ++k)
                        tma_load_2d(slot + k * K_REGION + lane * box * 128, &tmK, &full[i], h * HD + 64 * k, row);
                if (++i == slots) {
                    i = 0;
                    ph ^= 1;
                }
            }
        }
        if (lane == 0)                                 // every copy has landed before the CTA exits
            for (int j = max(it - slots, 0); j < it; ++j) mbar_wait(&full[j % slots], (j / slots) & 1, err, ERR_WAIT_PRODUCER);
    } else if (warp == 1) {
        const uint64_t d0 = sdesc_sw128(smem_u32(smem), 16, 1024);
        auto wait = [&](uint64_t *b, uint32_t parity) {
            return __all_sync(0xffffffffu, mbar_wait(b, parity, err, ERR_WAIT_MMA)) != 0;
        };
        int i = 0, buf = 0;
        uint32_t ph = 0, s_ph = 1;
        bool ok = true;
        while (ok && runs.next(s, L, r)) {
            const int N = (r.tokens * s.grp + 15) / 16 * 16;
            const uint32_t idesc = idesc_bf16(KW_TILE, 16, false, false) - ((16u >> 3) << 17) + ((uint32_t)(N >> 3) << 17);
            for (int h = 0; h < s.Hk; ++h) {
                if (!(ok = wait(&full[i], ph) && wait(&s_empty[buf], s_ph))) break;
                tc_fence_after();
                const uint64_t da = d0 + (uint64_t)((i * slot_bytes) >> 4), db = da + (uint64_t)(K_BYTES >> 4);
#pragma unroll
                for (int k = 0; k < NR; ++k)
                    key_issue4(tmem + buf * KST_COLS, da + (uint64_t)((k * K_REGION) >> 4), db + (uint64_t)((k * q_region) >> 4), idesc, k);
                tc_commit_warp(&empty[i]);
                tc_commit_warp(&s_full[buf]);
                if (++i == slots) {
                    i = 0;
                    ph ^= 1;
                }
                if (++buf == KST_BUFS) {
                    buf = 0;
                    s_ph ^= 1;
                }
            }
        }
        if (!ok) {                                     // a wait ran out: no product is under way when the CTA ends
            tc_commit_warp(drained);
            wait(drained, 0);
        }
    } else if (warp == 2) {
        // lse and limits of a step's columns, two a lane, read a step ahead of when they are stored
        int tk[2], gq[2], buf = 0, lim[2], lim_now[2];
        float nl[2];
        uint32_t ph = 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = lane + 32 * i;
            tk[i] = c / s.grp;
            gq[i] = c - tk[i] * s.grp;
        }
        auto read = [&](const KeyRun &x, int h) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                nl[i] = -INFINITY;
                lim[i] = 0;
                if (tk[i] < x.tokens) {
                    const int t = x.t0 + tk[i], b = t / s.n_q;
                    nl[i] = s.lse[(size_t)t * (s.Hk * s.grp) + h * s.grp + gq[i]];
                    lim[i] = min(max(s.limit(L.len[b], t - b * s.n_q) - x.key0, 0), KW_TILE);
                }
            }
        };
        int h = 0;
        bool ok = true, more = runs.next(s, L, r);
        if (more) read(r, h);
        while (ok && more) {
            float v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {              // a row that saw no key adds nothing
                v[i] = nl[i] == -INFINITY ? -INFINITY : -KW_LOG2E * nl[i];
                lim_now[i] = lim[i];
            }
            if (++h == s.Hk) {
                h = 0;
                more = runs.next(s, L, r);
            }
            if (more) read(r, h);
            ok = mbar_wait(&s_empty[buf], ph, err, ERR_WAIT_SOFTMAX);
            if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                cols[buf].nl[lane + 32 * i] = v[i];
                cols[buf].lim[lane + 32 * i] = lim_now[i];
            }
            mbar_arrive(&s_full[buf]);
            if (++buf == KST_BUFS) {
                buf = 0;
                ph ^= 1;
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, g = (warp - 4) >> 2, at = 32 * q + lane;         // key of the tile
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16);
        const float2 sl2 = make_float2(s.sl2, s.sl2);
        const int each = s.n_q * s.grp, place = s.nb * KW_TILE;
        int it = 0, tile = 0;
        bool ok = true;
        for (; ok && runs.next(s, L, r); ++tile) {
            const int n_br = r.own ? 1 : r.tokens / s.n_q, n_col = r.tokens * s.grp, p = tile & 1, key = r.key0 + at, it0 = it;
            float *mine = sums + (2 * p + g) * place + at;
            ok = __all_sync(0xffffffffu, mbar_wait(&taken[p], ((tile >> 1) & 1) ^ 1, err, ERR_WAIT_SOFTMAX)) != 0;
            if (!ok) break;
            // this group writes the tile: the old weights of eight branches are read ahead, those of more later
            float *w[8], old[8];
            auto read = [&](int j0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int b = r.own ? r.b : r.b * s.nb + j0 + j;
                    w[j] = j0 + j < n_br && key < r.end && key < L.len[b] ? s.w + (size_t)L.seq[b] * s.w_ld + key : nullptr;
                    old[j] = w[j] != nullptr && s.decay != 0.0f ? *w[j] : 0.0f;
                }
            };
            if ((tile & 1) == g) read(0);
            bool first = true;
            for (int h = 0; h < s.Hk; ++h, ++it) {
                if ((it & 1) != g) continue;
                const int buf = it & (KST_BUFS - 1);
                ok = mbar_wait(&s_full[buf], (it / KST_BUFS) & 1, err, ERR_WAIT_SOFTMAX);
                if (!(ok = __all_sync(0xffffffffu, ok) != 0)) break;
                tc_fence_after();
                const KeyCols &kc = cols[buf];
                const uint32_t from = lanes + buf * KST_COLS;
                auto put = [&](int j, float v) { mine[j * KW_TILE] = first ? v : mine[j * KW_TILE] + v; };
                auto exps = [&](int c, float *x) {     // of four columns from column c
                    const float4 nl = *reinterpret_cast<const float4 *>(&kc.nl[c]);
                    const int4 lim = *reinterpret_cast<const int4 *>(&kc.lim[c]);
                    const float2 a = __ffma2_rn(make_float2(x[0], x[1]), sl2, make_float2(nl.x, nl.y));
                    const float2 b = __ffma2_rn(make_float2(x[2], x[3]), sl2, make_float2(nl.z, nl.w));
                    x[0] = at < lim.x ? exp2_mufu(a.x) : 0.0f;
                    x[1] = at < lim.y ? exp2_mufu(a.y) : 0.0f;
                    x[2] = at < lim.z ? exp2_mufu(b.x) : 0.0f;
                    x[3] = at < lim.w ? exp2_mufu(b.y) : 0.0f;
                };
                auto run = [&](auto each_, auto n_) {  // branches of each_ columns, n_ in all
                    constexpr int E = decltype(each_)::value, n = decltype(n_)::value;
                    float x[n];
                    if constexpr (n == 64) tmem_ld64_sync(from, x);
                    else if constexpr (n == 48) {
                        tmem_ld32_sync(from, *reinterpret_cast<float (*)[32]>(x));
                        tmem_ld16_sync(from + 32, *reinterpret_cast<float (*)[16]>(x + 32));
                    } else if constexpr (n == 32) tmem_ld32_sync(from, x);
                    else tmem_ld16_sync(from, x);
#pragma unroll
                    for (int i = 0; i < n; i += 4) exps(i, x + i);
#pragma unroll
                    for (int j = 0; j < n / E; ++j) {
                        float sum = x[j * E];
#pragma unroll
                        for (int i = 1; i < E; ++i) sum += x[j * E + i];
                        if (j < n_br) put(j, sum);
                    }
                };
                auto pick = [&](auto each_) {
                    if (n_col <= 16) run(each_, std::integral_constant<int, 16>());
                    else if (n_col <= 32) run(each_, std::integral_constant<int, 32>());
                    else if (n_col <= 48) run(each_, std::integral_constant<int, 48>());
                    else run(each_, std::integral_constant<int, 64>());
                };
                switch (each) {
                    case 1: pick(std::integral_constant<int, 1>()); break;
                    case 2: pick(std::integral_constant<int, 2>()); break;
                    case 3: pick(std::integral_constant<int, 3>()); break;
                    case 4: pick(std::integral_constant<int, 4>()); break;
                    case 5: pick(std::integral_constant<int, 5>()); break;
                    case 6: pick(std::integral_constant<int, 6>()); break;
                    case 7: pick(std::integral_constant<int, 7>()); break;
                    case 8: pick(std::integral_constant<int, 8>()); break;
                    default: {
                        float sum = 0.0f;
                        int left = each, j = 0;        // columns of branch j still to come
                        for (int c = 0; c < n_col; c += 16) {
                            float x[16];
                            tmem_ld16_sync(from + c, x);
#pragma unroll
                            for (int i = 0; i < 16; i += 4) exps(c + i, x + i);
                            if (left > 16) {
                                float2 t = make_float2(x[0], x[1]);
#pragma unroll
                                for (int i = 2; i < 16; i += 2) t = __fadd2_rn(t, make_float2(x[i], x[i + 1]));
                                sum += t.x + t.y;
                                left -= 16;
                                continue;
                            }
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                sum += x[i];
                                if (--left == 0) {
                                    if (j < n_br) put(j, sum);
                                    sum = 0.0f;
                                    left = each;
                                    ++j;
                                }
                            }
                        }
                    }
                }
                first = false;
                tc_fence_before();
                mbar_arrive(&s_empty[buf]);
            }
            if (!ok) break;
            mbar_arrive(&added[p]);
            if ((tile & 1) != g) continue;
            const float *sum0 = sums + 2 * p * place + at, *sum1 = sum0 + place;
            const bool in0 = s.Hk > 1 || (it0 & 1) == 0, in1 = s.Hk > 1 || (it0 & 1) == 1;        // groups that had a step
            for (int j0 = 0; j0 < n_br; j0 += 8) {
                if (j0 > 0) read(j0);
                if (j0 == 0 && !(ok = __all_sync(0xffffffffu, mbar_wait(&added[p], (tile >> 1) & 1, err, ERR_WAIT_SOFTMAX)) != 0)) break;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (w[j] != nullptr) {
                        const int from = (j0 + j) * KW_TILE;
                        const float v = (in0 ? sum0[from] : 0.0f) + (in1 ? sum1[from] : 0.0f);
                        *w[j] = s.decay == 0.0f ? v : fmaf(s.decay, old[j], v);
                    }
            }
            mbar_arrive(&taken[p]);
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

// ------------------------------------------------------------ fp32 kernel
// 64 keys x 64 rows at a time, 256 threads as 16 x 16: thread (ty, tx) has rows 4 ty..
// and keys tx + 16 j.  A unit is 64 keys with all their rows, taken in turn; the C CTAs of a
// cluster have every C-th key head of it, and the first one adds their sums in order and writes them
// (C = 4 at most: 4 x 232 queries over 696 keys, 4 heads x 16, 15.6 us instead of 35.6 with one CTA a unit;
// 4 single tokens, 8 heads x 64, 1088 keys 18.9 instead of 40.2, with eight 22.0).
constexpr int KF_KEYS = 64;
__device__ __forceinline__ float cluster_read(const float *p, int rank) {     // the same place of another CTA's shared memory
    unsigned at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
template <int HD, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(256)
    key_weights_f32_kernel(const float *__restrict__ q, const long q_ld, const float *__restrict__ k,
                           const __grid_constant__ KeySched s, int *err) {
    constexpr int LD = HD + 4;
    extern __shared__ __align__(16) float sm[];
    __shared__ KeyLens L;
    __shared__ float sh_nl[64], sh_out[64];
    __shared__ int sh_lim[64];
    float *sK = sm, *sQ = sm + 64 * LD;
    const int rank = blockIdx.x % C;
    pdl_wait();
    pdl_release();
    key_lens<false>(s, L, KF_KEYS, err);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, log_ps = 31 - __clz(s.ps), rows = s.n_q * s.grp;
    const float scale = s.sl2;
    int b = 0, before = 0;                             // units of the branches before b
    for (int u = blockIdx.x / C;; u += gridDim.x / C) {
        while (b < s.B && u - before >= key_tiles(s, L.len[b], KF_KEYS)) {
            before += key_tiles(s, L.len[b], KF_KEYS);
            ++b;
        }
        if (b == s.B) return;                          // (all of a cluster at the same time)
        const int key0 = (u - before) * KF_KEYS, l = L.len[b], seq = L.seq[b];
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int h = rank; h < s.Hk; h += C) {
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
        float v = 0.0f;
        if (tid < 64)
            for (int y = 0; y < 16; ++y) v += sm[y * 64 + tid];
        if constexpr (C > 1) {
            if (tid < 64) sh_out[tid] = v;
            asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
            if (rank == 0 && tid < 64)
                for (int c = 1; c < C; ++c) v += cluster_read(&sh_out[tid], c);
            // no CTA writes its next sums, or ends, before the first has read these
            asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
        }
        if (rank == 0 && tid < 64 && key0 + tid < l) s.put(seq, key0 + tid, v);
    }
}

// ------------------------------------------------------------------- host
static size_t few_smem(int Hk, int N, int head_dim) { return (size_t)Hk * N * (head_dim * 2 + 4) + 2 * (size_t)KFEW_WARPS * N * KFEW_PITCH * 4; }
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
    const long long each = (long long)n_q * s.grp;
    auto fits = [&](long long n) { return n * each <= KFEW_COLS && few_smem(s.Hk, (int)(n * each + 7) / 8 * 8, c.head_dim) <= KFEW_SMEM; };
    const long long keys = (long long)c.max_pages * c.page_size, most = shared > 0 && B > 1 ? shared + B * (keys - shared) : B * keys;
    if (each <= KST_COLS && (!fits(1) || most * s.Hk * c.head_dim * 2 > KST_BYTES)) {      // few rows, many keys
        if (shared > 0 && B > 1) {
            while (s.nb < std::min(B, KST_NB) && (s.nb + 1) * each <= KST_COLS) ++s.nb;
            s.P = shared;
        }
        s.stream = 1;
        s.tt = s.nb * n_q;
        s.N = (s.tt * s.grp + 15) / 16 * 16;
        s.n_ct = (B + s.nb - 1) / s.nb;
        s.n_pt = (s.P + KW_TILE - 1) / KW_TILE;
        return s;
    }
    if (fits(1)) {                                     // few rows
        s.wh = 1;
        while (s.wh < KFEW_WARPS && s.wh < s.Hk) s.wh *= 2;
        s.wk = KFEW_WARPS / s.wh;
        if (shared > 0 && B > 1) {
            while (s.nb < B && fits(s.nb + 1)) ++s.nb;
            s.P = shared;
        }
        s.tt = s.nb * n_q;
        s.N = (s.tt * s.grp + 7) / 8 * 8;
        s.n_ct = (B + s.nb - 1) / s.nb;
        s.n_pt = (s.P + 16 * s.wk - 1) / (16 * s.wk);
        return s;
    }
    s.tt = std::min(KW_COLS / s.grp, n_q);
    s.N = (s.tt * s.grp + 15) / 16 * 16;
    s.n_ct = (n_q + s.tt - 1) / s.tt;
    return s;
}
bool key_weights_fit(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    const KeySched s = key_plan(c, B, n_q, H, shared);
    const long long tiles = ((long long)c.max_pages * c.page_size + 15) / 16 + 1;
    return B <= KW_MAX_B && tiles * B * s.Hk * s.n_ct < (1ll << 31);
}
size_t key_weights_workspace_bytes(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    const KeySched s = key_plan(c, B, n_q, H, shared);
    return c.dtype == XC_F32 || s.wh > 0 || s.stream ? 16 : (size_t)2 * s.G * (sizeof(int4) + KW_KEYS * sizeof(float));
}

template <int HD>
static cudaError_t key_launch_tc(const xc_kv_cache &c, const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    constexpr int K_BYTES = KW_TILE * HD * 2, BUDGET = 192 * 1024;
    static DeviceSet asked{0};
    cudaError_t e = allow_smem(key_weights_kernel<HD>, BUDGET + 1024, asked);
    if (e != cudaSuccess) return e;
    const int q_bytes = s.N * HD * 2;
    const int q_slots = std::min(8, (BUDGET - 2 * K_BYTES) / q_bytes);
    const uint64_t rows = (uint64_t)c.n_pages * c.page_size, cols = (uint64_t)c.n_kv_heads * HD;
    CUtensorMap tq, tk;
    if (!make_tmap_heads_bf16(&tq, a.q, HD, (uint64_t)s.Hk * s.grp, (uint64_t)s.B * s.n_q, a.q_ld, s.grp, s.tt) ||
        !make_tmap_bf16(&tk, a.k, rows, cols, c.page_size < KW_TILE ? c.page_size : KW_TILE))
        return cudaErrorInvalidValue;
    e = launch_pdl(key_weights_kernel<HD>, dim3(s.G), dim3(KW_THREADS),
                   2 * K_BYTES + q_slots * q_bytes + 1024, st, tq, tk, s, q_slots, err);
    if (e != cudaSuccess) return e;
    return launch_pdl(key_merge_kernel, dim3(2 * s.G), dim3(KW_KEYS), 0, st, s);
}
template <int HD>
static cudaError_t key_launch_stream(const xc_kv_cache &c, const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    static DeviceSet asked{0};
    const cudaError_t e = allow_smem(key_weights_stream_kernel<HD>, KST_BUDGET + 1024, asked);
    if (e != cudaSuccess) return e;
    const int slot = (KW_TILE + s.N) * HD * 2, sums = 4 * s.nb * KW_TILE * 4, slots = std::min(KST_SLOTS, (KST_BUDGET - sums) / slot);
    const uint64_t rows = (uint64_t)c.n_pages * c.page_size, cols = (uint64_t)c.n_kv_heads * HD;
    CUtensorMap tq, tk;
    if (!make_tmap_heads_bf16(&tq, a.q, HD, (uint64_t)s.Hk * s.grp, (uint64_t)s.B * s.n_q, a.q_ld, s.grp, s.tt) ||
        !make_tmap_bf16(&tk, a.k, rows, cols, std::min(s.ps, KW_TILE)))
        return cudaErrorInvalidValue;
    return launch_pdl(key_weights_stream_kernel<HD>, dim3(s.G), dim3(KST_THREADS), slots * slot + sums + 1024, st, tq, tk, s, slots, err);
}
template <int HD, int NT>
static cudaError_t key_launch_few(const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    if constexpr (NT > 1)
        if (s.N < 8 * NT) return key_launch_few<HD, NT - 1>(a, s, err, st);
    static DeviceSet asked{0};
    const cudaError_t e = allow_smem(key_weights_few_kernel<HD, NT>, (int)KFEW_SMEM, asked);
    if (e != cudaSuccess) return e;
    return launch_pdl(key_weights_few_kernel<HD, NT>, dim3(s.G), dim3(KFEW_THREADS), few_smem(s.Hk, s.N, HD), st,
                      reinterpret_cast<const bf16 *>(a.q), a.q_ld, reinterpret_cast<const bf16 *>(a.k), s, err);
}
template <int HD, int C>
static cudaError_t key_launch_f32(const KeyWeightsArgs &a, const KeySched &s, int *err, cudaStream_t st) {
    if constexpr (C > 1)
        if (s.Hk < C) return key_launch_f32<HD, C / 2>(a, s, err, st);
    constexpr int SMEM = 2 * 64 * (HD + 4) * 4;
    static DeviceSet asked{0};
    if (SMEM > 48 * 1024) {
        const cudaError_t e = allow_smem(key_weights_f32_kernel<HD, C>, SMEM, asked);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(key_weights_f32_kernel<HD, C>, dim3(4 * s.G / C * C), dim3(256), SMEM, st, reinterpret_cast<const float *>(a.q), a.q_ld,
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
        if (c.head_dim == 64) return s.stream ? key_launch_stream<64>(c, a, s, err, st) : s.wh > 0 ? key_launch_few<64, KFEW_COLS / 8>(a, s, err, st) : key_launch_tc<64>(c, a, s, err, st);
        if (c.head_dim == 128) return s.stream ? key_launch_stream<128>(c, a, s, err, st) : s.wh > 0 ? key_launch_few<128, KFEW_COLS / 8>(a, s, err, st) : key_launch_tc<128>(c, a, s, err, st);
        return cudaErrorInvalidValue;
    }
    switch (c.head_dim) {
        case 16: return key_launch_f32<16, 4>(a, s, err, st);
        case 32: return key_launch_f32<32, 4>(a, s, err, st);
        case 64: return key_launch_f32<64, 4>(a, s, err, st);
        case 128: return key_launch_f32<128, 4>(a, s, err, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace xc
