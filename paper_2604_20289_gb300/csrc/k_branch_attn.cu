// Attention of a batch of branches over a paged cache whose first part they
// share.
//
//   o[t] = sum_j p_j v_j, p = softmax_j(scale q[t] . k_j), j < limit(t)
//
// A unit is (key head, row tile, key range).  Row tiles hold tt consecutive
// tokens x the group's query heads.  With prefix units the shared keys are
// read for tiles packed over ALL branches' rows, and every branch's own keys
// for tiles of its own rows; without them (one branch, or branches whose rows
// fill tiles by themselves) a unit reads its branch's whole sequence.  The
// key tiles of all units, head by head, form one line that the CTAs share
// evenly, whatever the branches' lengths: each CTA finds its start by a scan
// over the lengths.  A piece of a unit leaves its unnormalised O with the
// running max m (log2 units) and sum l,
//   O = sum_j 2^(s_j - m) v_j,   l = sum_j 2^(s_j - m),
// and branch_combine_kernel adds the pieces of a row in a fixed order,
//   o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p,   M = max_p m_p;
// a row whose unit one CTA ran whole, without prefix units, is written at once.
#include "xc_branch.cuh"
#include "xc_ptx.cuh"

namespace xc {

constexpr int LEN_CACHE = 64;    // branches whose table row and length are kept in shared memory

struct BranchSched {
    int B, n_q, grp, Hk;
    int tt;                  // tokens of a row tile
    int n_pr, n_pt;          // prefix row tiles and key tiles (n_pr = 0: no prefix units)
    int n_st, E;             // own row tiles per branch, of all branches
    int P;                   // keys of the prefix units: own keys begin there
    int shared;              // the caller's shared_len, which no sequence may be shorter than
    int causal, G;           // G: CTAs
    int lead;                // what a unit costs beside its key tiles, in key tiles (see branch_plan)
    int max_seqs, max_pages, ps, n_pages;
    int pitch_p, pitch_o;    // rows of a partial slot
    long slots_p;            // prefix slots before the own ones
    const int *seqs, *len, *table;
    float *ws_o;             // partial O, then (m, l) of each row, then the scan
    float2 *ws_ml;
    int *ws_off;             // [E + 1] line length before each entry (same for every head)
    float *lse;              // [B n_q][Hk grp] log of each row's sum of exponentials, or NULL
    int4 *ws_start;          // [G] per CTA: its first unit (head, entry), position in it, key tiles of it

    __host__ __device__ __forceinline__ int seq(int b) const {
        const int s = seqs[b];
        return s >= 0 && s < max_seqs ? s : -1;
    }
    __host__ __device__ __forceinline__ int load_len(int b) const {
        const int s = seq(b);
        const int l = s < 0 ? 0 : len[s];
        return l < 0 || l > max_pages * ps ? 0 : l;
    }
    __host__ __device__ __forceinline__ int seq_len(int b, const int *cache) const {
        return b < LEN_CACHE ? cache[b] : load_len(b);
    }
    __host__ __device__ __forceinline__ int table_row(int b, const int *cache) const {
        return b < LEN_CACHE ? cache[LEN_CACHE + b] : seq(b);
    }
    // length on the line of a unit of n key tiles
    __host__ __device__ __forceinline__ int line_len(int n) const { return n > 0 ? n + lead : 0; }
    // log sum_j exp(scale q . k_j) of a row, from its max m (log2 units) and sum l: -inf without keys
    // (no term: l = 0).  l is NaN where a score is NaN (m passes over those) and where the
    // largest is +inf, whose weight is 2^(inf - inf): m is +inf then, and so is the log.
    __device__ __forceinline__ void put_lse(int t, int head, float m, float l) const {
        const float y = l == 0.0f ? -INFINITY : m == INFINITY ? INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        lse[(size_t)t * (Hk * grp) + head] = y;
    }
    // keys that query i of a branch of length l sees
    __host__ __device__ __forceinline__ int limit(int l, int i) const {
        const int x = causal ? l - n_q + i + 1 : l;
        return x > 0 ? x : 0;
    }
    // keys past P that the last row of entry (branch b, row tile j) sees
    __host__ __device__ __forceinline__ int own_keys(int b, int j, const int *cache) const {
        return max(limit(seq_len(b, cache), min((j + 1) * tt, n_q) - 1) - P, 0);
    }
    __host__ __device__ __forceinline__ int own_keys(int e, const int *cache) const {
        return own_keys(e / n_st, e % n_st, cache);
    }
};

// The line of length T (< 2^31) over G CTAs: CTA c runs [begin(c),
// begin(c + 1)), lengths that differ by one at most.  Key tile k of a unit
// that begins at x sits at x + lead + k.
struct BranchLine {
    unsigned q, r;
    __host__ __device__ __forceinline__ BranchLine(unsigned T, unsigned G) : q(T / G), r(T - q * G) {}
    __host__ __device__ __forceinline__ unsigned begin(unsigned c) const { return q * c + (c < r ? c : r); }
    __host__ __device__ __forceinline__ unsigned owner(unsigned x) const {   // the c with begin(c) <= x < begin(c + 1)
        const unsigned longer = r * (q + 1);
        return x < longer ? x / (q + 1) : r + (x - longer) / q;
    }
};

// One piece of a unit, as every role of a CTA walks them.
struct BranchPiece {
    int h, t0, nt;           // key head, first token row, tokens
    int b;                   // branch whose table row holds the keys
    int key0, keys;          // first key and keys of the unit
    int kt0, kt1, n_kt;      // key tiles of the piece and of the unit
    int first;               // key tile that the tensor-core kernel begins with
    int idx;                 // unit of the head: prefix tiles, then entries
};
struct BranchStart {
    int h, idx, off, n;      // first unit, position in it, line length of this CTA
};

//
// Order of the key tiles.  A softmax may take its keys in any order, so CTAs
// that read the same keys take them in step, and one read from DRAM serves all
// of them through L2: after `done` key tiles a CTA begins a whole unit of n at
// tile done mod n and goes around.  A cut unit's tiles count from its end, so
// that the CTA it is cut to -- whose clock is at 0 -- begins at tile 0, and all
// CTAs end at tile n - 1.
template <int KT>
struct BranchWalk {
    int h, idx, off, left, done;
    int b, j;                // entry idx - n_pr (idx >= n_pr)
    BranchWalk() = default;
    __host__ __device__ __forceinline__ BranchWalk(const BranchSched &s, const BranchStart &st)
        : h(st.h), idx(st.idx), off(st.off), left(st.n), done(0) {
        const int e = max(idx - s.n_pr, 0);
        b = e / s.n_st;
        j = e - b * s.n_st;
    }
    __host__ __device__ __forceinline__ bool next(const BranchSched &s, const int *lens, BranchPiece &p) {
        while (left > 0) {
            const bool own = idx >= s.n_pr;
            const int keys = own ? s.own_keys(b, j, lens) : s.P;
            const int n = own ? (keys + KT - 1) / KT : s.n_pt, len = s.line_len(n);
            if (off < len) {
                const int end = min(len, off + left);
                p.n_kt = n;
                p.h = h;
                p.idx = idx;
                p.keys = keys;
                p.b = own ? b : 0;
                p.t0 = own ? b * s.n_q + j * s.tt : idx * s.tt;
                p.nt = min(s.tt, own ? s.n_q - j * s.tt : s.B * s.n_q - p.t0);
                p.key0 = own ? s.P : 0;
                p.kt0 = max(off - s.lead, 0);
                p.kt1 = max(end - s.lead, 0);
                left -= end - off;
                off = end;
                if (p.kt1 > p.kt0) {
                    p.first = p.kt1 - p.kt0 == n ? done % n : n - p.kt1;
                    done += p.kt1 - p.kt0;
                    return true;
                }
                continue;
            }
            off = 0;
            if (own && ++j == s.n_st) {
                j = 0;
                ++b;
            }
            if (++idx == s.n_pr + s.E) {
                idx = 0;
                b = 0;
                ++h;
            }
        }
        return false;
    }
};

// This CTA's share of the line.  Every thread calls it; lens (2 LEN_CACHE ints)
// receives the branches' lengths, then their table rows.
template <int KT>
__device__ BranchStart branch_start(const BranchSched &s, int *lens, int *sh, BranchStart *out) {
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = nt >> 5;
    const int c = blockIdx.x;
    for (int b = tid; b < min(s.B, LEN_CACHE); b += nt) {
        lens[b] = s.load_len(b);
        lens[LEN_CACHE + b] = s.seq(b);
    }
    if (tid == 0) out->n = 0;
    __syncthreads();
    const int per = (s.E + nt - 1) / nt;
    const int e0 = min(tid * per, s.E), e1 = min(e0 + per, s.E);
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += s.line_len((s.own_keys(e, lens) + KT - 1) / KT);
    int x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    int before = 0, S = 0;
    for (int w = 0; w < nw; ++w) {
        if (w < warp) before += sh[w];
        S += sh[w];
    }
    const int excl = before + x - mine;
    const unsigned PP = (unsigned)s.n_pr * s.line_len(s.n_pt), Th = PP + S, T = Th * s.Hk;
    const BranchLine line(T, s.G);
    const unsigned g0 = line.begin(c), g1 = line.begin(c + 1);
    if (g1 > g0) {
        const unsigned h = g0 / Th, r = g0 - h * Th;
        if (r < PP) {
            const int len = s.line_len(s.n_pt);
            if (tid == 0) *out = BranchStart{(int)h, (int)r / len, (int)r % len, (int)(g1 - g0)};
        } else if ((int)(r - PP) >= excl && (int)(r - PP) < excl + mine) {
            int rest = (int)(r - PP) - excl, e = e0, n;
            for (;; ++e) {
                n = (s.own_keys(e, lens) + KT - 1) / KT;
                if (rest < s.line_len(n)) break;
                rest -= s.line_len(n);
            }
            *out = BranchStart{(int)h, s.n_pr + e, rest, (int)(g1 - g0)};
            s.ws_start[c] = make_int4(h, e, rest, n);
        }
    }
    __syncthreads();
    return *out;
}

// One warp of one CTA: the entries' scan for the combine kernel, and a check of
// what the host could not see.
template <int KT>
__device__ void branch_publish(const BranchSched &s, const int *lens, int *err) {
    const int lane = threadIdx.x & 31;
    int base = 0;
    for (int e0 = 0; e0 < s.E; e0 += 32) {
        const int e = e0 + lane;
        const int mine = e < s.E ? s.line_len((s.own_keys(e, lens) + KT - 1) / KT) : 0;
        int x = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (e < s.E) s.ws_off[e] = base + x - mine;
        base += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) s.ws_off[s.E] = base;
    for (int b = lane; b < s.B; b += 32) {
        const int q = s.seqs[b];
        if (err && (q < 0 || q >= s.max_seqs || s.len[q] < 0 || s.len[q] > s.max_pages * s.ps || s.len[q] < s.shared))
            atomicOr(err, ERR_BAD_SEQ);
    }
}

// Entries without a key to read: their rows are zero (with prefix units the
// combine kernel writes every row).
template <typename T>
__device__ void branch_zero_rows(const BranchSched &s, const int *lens, T *o, long o_ld, int d) {
    if (s.n_pr > 0) return;
    for (int e = blockIdx.x; e < s.E; e += s.G) {
        if (s.own_keys(e, lens) > 0) continue;
        const int b = e / s.n_st, i0 = (e % s.n_st) * s.tt, nt = min(s.tt, s.n_q - i0);
        const int vecs = d * (int)sizeof(T) / 16;
        for (int x = threadIdx.x; x < nt * vecs; x += blockDim.x)
            reinterpret_cast<uint4 *>(o + (size_t)(b * s.n_q + i0 + x / vecs) * o_ld)[x % vecs] = make_uint4(0, 0, 0, 0);
        if (s.lse != nullptr)
            for (int x = threadIdx.x; x < nt * s.Hk * s.grp; x += blockDim.x)
                s.lse[(size_t)(b * s.n_q + i0) * (s.Hk * s.grp) + x] = -INFINITY;
    }
}

// Partial slot of a piece (its first row): with prefix units, unit index + CTA
// (both only grow along the line, so the sum names the piece); without, a
// CTA cuts at most its first and its last unit.  A slot holds its O by
// 4-column chunks, [HD / 4][pitch rows][4]: threads that hold neighbouring
// rows write neighbouring 16 bytes.
__host__ __device__ __forceinline__ long branch_slot_row(const BranchSched &s, const BranchPiece &p, int c, bool first) {
    if (s.n_pr > 0)
        return p.idx < s.n_pr ? ((long)p.h * s.n_pr + p.idx + c) * s.pitch_p
                              : s.slots_p * s.pitch_p + ((long)p.h * s.E + (p.idx - s.n_pr) + c) * s.pitch_o;
    return (2l * c + (first ? 0 : 1)) * s.pitch_o;
}

// ------------------------------------------------------- tensor-core kernel
template <int HD_, int QT_>
struct BranchTile {
    static constexpr int HD = HD_, QT = QT_;
    static constexpr int NR = HD / 64;                 // 64-wide swizzle regions per row
    static constexpr int REGION = 128 * 128;           // [128 rows][64 bf16]
    static constexpr int Q_BYTES = NR * REGION, KV_BYTES = NR * REGION;
    // K and V tiles share a ring of SLOTS in the order K0 V0 K1 V1 ...: as many
    // as fit beside Q (with 2 + 2 slots instead of 5 the loads of a tile were
    // requested one tile before its use, about the latency under load).
    static constexpr int SLOTS = HD == 64 ? 10 : (QT == 2 ? 5 : 6);
    static constexpr int PAIRS = 8;                    // barriers of (V_g, K_g+1), more than the ring can hold
    static constexpr int OFF_KV = QT * Q_BYTES, OFF_BAR = OFF_KV + SLOTS * KV_BYTES;
    static constexpr int SMEM_BYTES = OFF_BAR + 448 + 1024;
    static constexpr bool SEP_P = HD == 64 || QT == 1;     // P has TMEM columns of its own
    static constexpr int ISSUERS = SEP_P ? QT : 1;
    static constexpr int S_COL(int i) { return 128 * i; }
    static constexpr int O_COL(int i) { return 128 * QT + HD * i; }
    static constexpr int P_COL(int i) { return SEP_P ? QT * (128 + HD) + 64 * i : 128 * i; }
    static constexpr int TMEM_COLS = HD == 64 && QT == 1 ? 256 : 512;
    static constexpr int W_TMA = 4 * QT, W_MMA = W_TMA + 1, W_TAIL = W_MMA + ISSUERS;
    static constexpr int THREADS = 32 * (W_TAIL + 1);
    static constexpr bool TURNS = HD == 64 && QT == 2;
    static constexpr float LAZY = 8.0f;                // rescale threshold (log2 units)
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// 4 x 4 transpose of 16-byte parts within each quad of lanes: lane i's u[j]
// becomes lane j's u[i].
__device__ __forceinline__ uint4 shfl_xor16(const uint4 &v, int d) {
    return make_uint4(__shfl_xor_sync(0xffffffffu, v.x, d), __shfl_xor_sync(0xffffffffu, v.y, d),
                      __shfl_xor_sync(0xffffffffu, v.z, d), __shfl_xor_sync(0xffffffffu, v.w, d));
}
__device__ __forceinline__ uint4 pick16(bool c, const uint4 &a, const uint4 &b) {
    return make_uint4(c ? a.x : b.x, c ? a.y : b.y, c ? a.z : b.z, c ? a.w : b.w);
}
__device__ __forceinline__ void quad_transpose(uint4 (&u)[4], int lane) {
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const bool hi = lane & 1;
        const uint4 got = shfl_xor16(pick16(hi, u[k], u[k + 1]), 1);
        u[k] = pick16(hi, got, u[k]);
        u[k + 1] = pick16(hi, u[k + 1], got);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const bool hi = lane & 2;
        const uint4 got = shfl_xor16(pick16(hi, u[k], u[k + 2]), 2);
        u[k] = pick16(hi, got, u[k]);
        u[k + 2] = pick16(hi, u[k + 2], got);
    }
}

struct BranchWarpWalk {
    BranchWalk<128> w;
    BranchPiece pc[2];       // piece p of the CTA in slot p & 1
    int more;                // whether the piece walked to last exists
};

// Warps: 4 QT softmax (thread = row of a 128-row tile = TMEM lane), one that
// loads (Q of a piece, then 128-key K and V tiles, page by page, by TMA), the
// MMA issuers (one per row tile where P has its own TMEM columns, else one),
// and one that clears the value rows past a unit's last key, whose weights are
// zero but whose bytes may be anything.
// Measured, with the merge: 2 x 4320 queries over 30240 keys, 12 heads x 128,
// 1008-1030 us back to back (1.6 PFLOP/s, at the power cap), 913-929 after a pause
// with the tensor pipe 76 % busy (2620 cycles a key tile of 256 rows); the same of
// 12 heads x 64, 728 us; 32 single tokens over 38880 shared + 1..1500 own keys, 40 / 8 heads
// x 128, 63 us for 258 MB, of which 7 until the first tile and 7 the merge.  Where
// units are short the latency of a piece bounds it: 200 single tokens over 256 +
// 16..120 keys, 32 / 8 heads x 128, 62 us, 10 or 11 pieces of one key tile a CTA at
// about 4 us (queries, S, softmax, P V and output one after another).
template <int HD, int QT>
__global__ void __launch_bounds__(BranchTile<HD, QT>::THREADS, 1)
    branch_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, bf16 *o, const long o_ld, const float sl2,
                       const int tt1, const __grid_constant__ BranchSched sc, int *err) {
    using A = BranchTile<HD, QT>;
    static_assert(A::SMEM_BYTES + sizeof(BranchWarpWalk) * 4 * QT + 4 * (2 * LEN_CACHE + 16) + 32 <= 232448,
                  "227 KB of shared memory a CTA");
    extern __shared__ uint8_t smem_raw[];
    __shared__ int sh_len[2 * LEN_CACHE], sh_scan[16];
    __shared__ BranchStart sh_start;
    __shared__ BranchWarpWalk sh_walk[4 * QT];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t *sQ = smem, *sKV = smem + A::OFF_KV;
    uint64_t *bar = reinterpret_cast<uint64_t *>(smem + A::OFF_BAR);
    uint64_t *q_full = bar;                    // Q of piece p landed
    uint64_t *q_empty = bar + 1;               // every S of piece p done
    uint64_t *k0_full = bar + 2;               // the first K tile landed
    uint64_t *pair = bar + 3;                  // [PAIRS] V_g (cleared past the last key) and K_g+1 landed
    uint64_t *v_tail = pair + A::PAIRS;        // [PAIRS] V_g landed, where it is to be cleared
    uint64_t *empty = v_tail + A::PAIRS;       // [SLOTS] slot read by every issuer
    uint64_t *s_full = empty + A::SLOTS;       // [QT] S_i computed
    uint64_t *s_cons = s_full + QT;            // [QT] S_i read (SEP_P)
    uint64_t *p_full = s_cons + QT;            // [QT] P_i written, O_i corrected
    uint64_t *p_half = p_full + QT;            // [QT] first 64 keys of P_i written, O_i corrected (SEP_P)
    uint64_t *pv_done = p_half + QT;           // [QT] P_i V done (SEP_P: every tile; else last of a piece)
    uint64_t *o_free = pv_done + QT;           // [QT] O_i of piece p read out
    uint64_t *turn = o_free + QT;              // [2][4] exponential-phase hand-off (TURNS)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(turn + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, A::ISSUERS);
        mbar_init(k0_full, 1);
        for (int s = 0; s < A::PAIRS; ++s) {
            mbar_init(&pair[s], 2);
            mbar_init(&v_tail[s], 1);
        }
        for (int s = 0; s < A::SLOTS; ++s) mbar_init(&empty[s], A::ISSUERS);
        for (int i = 0; i < QT; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_cons[i], 128);
            mbar_init(&p_full[i], 128);
            mbar_init(&p_half[i], 128);
            mbar_init(&pv_done[i], 1);
            mbar_init(&o_free[i], 128);
        }
        for (int i = 0; i < 8; ++i) mbar_init(&turn[i], 1);
        mbar_fence_init();
    }
    if (warp == A::W_MMA) tmem_alloc(tmem_slot, A::TMEM_COLS);
    // nothing above depends on the kernels before this one
    pdl_wait();
    const BranchStart start = branch_start<128>(sc, sh_len, sh_scan, &sh_start);
    branch_zero_rows<bf16>(sc, sh_len, o, o_ld, sc.Hk * sc.grp * HD);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (blockIdx.x == 0 && warp == A::W_TAIL) branch_publish<128>(sc, sh_len, err);
    BranchWalk<128> walk(sc, start);
    BranchPiece pc;

    if (start.n == 0) {
        // a line shorter than the CTAs are many
    } else if (warp == A::W_TMA) {
        // ------------------------------------------------------ TMA producer
        const int box = min(sc.ps, 128), log_ps = 31 - __clz(sc.ps);
        const int q_bytes = QT * A::NR * tt1 * sc.grp * 128;
        int p = 0, g = 0;
        int slot = 0;
        uint32_t turn_ph = 0;                  // parity of the ring's turn
        uint32_t tails = 0, tail_ph = 0;       // pairs whose last use was a tail, parity of their tail uses
        bool ok = true;
        while (ok && walk.next(sc, sh_len, pc)) {
            if (p > 0) ok = mbar_wait(q_empty, (p - 1) & 1, err, ERR_WAIT_PRODUCER);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(q_full, q_bytes);
                for (int i = 0; i < QT; ++i)
                    for (int r = 0; r < A::NR; ++r)
                        tma_load_3d(sQ + i * A::Q_BYTES + r * A::REGION, &tmQ, q_full, 64 * r, pc.h * sc.grp,
                                    pc.t0 + i * tt1);
            }
            ++p;
            const int row_id = sc.table_row(pc.b, sh_len);
            const int *pages = sc.table + (size_t)max(row_id, 0) * sc.max_pages;
            // first pool row of this lane's page in key tile kt (lane < pages of a tile)
            auto page_row = [&](int kt) {
                const int key = pc.key0 + kt * 128 + lane * box;
                if (lane * box >= 128 || kt * 128 + lane * box >= pc.keys) return -1;
                const int id = row_id < 0 ? -1 : pages[key >> log_ps];   // (a prefix unit of a bad first sequence)
                if (id < 0 || id >= sc.n_pages) {
                    if (err) atomicOr(err, ERR_BAD_SEQ);
                    return sc.n_pages * sc.ps;         // out of range: TMA fills zeros
                }
                return id * sc.ps + (key & (sc.ps - 1));
            };
            int kt = pc.first, nrow = page_row(kt);
            for (int i = pc.kt1 - pc.kt0; i > 0; --i, ++g) {
                const int row = nrow;
                const bool tail = pc.keys < (kt + 1) * 128;
                kt = kt + 1 == pc.n_kt ? 0 : kt + 1;
                if (i > 1) nrow = page_row(kt);
                const int n_pg = __popc(__ballot_sync(0xffffffffu, row >= 0));
                const uint32_t bytes = n_pg * box * 128 * A::NR;
                auto load = [&](const CUtensorMap *tm, uint64_t *b) -> bool {      // the next slot
                    const bool r = mbar_wait(&empty[slot], turn_ph ^ 1, err, ERR_WAIT_PRODUCER);
                    if (!__all_sync(0xffffffffu, r)) return false;
                    if (lane == 0) mbar_expect_tx(b, bytes);
                    __syncwarp();
                    if (row >= 0)
                        for (int r2 = 0; r2 < A::NR; ++r2)
                            tma_load_2d(sKV + slot * A::KV_BYTES + r2 * A::REGION + lane * box * 128, tm, b,
                                        pc.h * HD + 64 * r2, row);
                    if (++slot == A::SLOTS) {
                        slot = 0;
                        turn_ph ^= 1;
                    }
                    return true;
                };
                const int pi = g % A::PAIRS;
                ok = load(&tmK, g == 0 ? k0_full : &pair[(g - 1) % A::PAIRS]);
                if (!ok) break;
                ok = load(&tmV, tail ? &v_tail[pi] : &pair[pi]);
                if (!ok) break;
                if (tail) tail_ph ^= 1u << pi;
                tails = tail ? tails | 1u << pi : tails & ~(1u << pi);
            }
        }
        // every copy this warp started has landed before the CTA exits
        if (lane == 0) {
            if (g > 0) {
                mbar_arrive(&pair[(g - 1) % A::PAIRS]);        // the last V tile is not followed by a K tile
                mbar_wait(k0_full, 0, err, ERR_WAIT_PRODUCER);
            }
            if (p > 0) mbar_wait(q_full, (p - 1) & 1, err, ERR_WAIT_PRODUCER);
            for (int x = max(g - A::PAIRS, 0); x < g; ++x) {
                const int pi = x % A::PAIRS;
                if (tails >> pi & 1u) mbar_wait(&v_tail[pi], (tail_ph >> pi & 1u) ^ 1u, err, ERR_WAIT_PRODUCER);
                mbar_wait(&pair[pi], (x / A::PAIRS) & 1, err, ERR_WAIT_PRODUCER);
            }
        }
    } else if (warp == A::W_TAIL) {
        // -------------------------------- clears V rows past the last key
        uint32_t ph = 0;
        int g = 0;
        bool ok = true;
        while (ok && walk.next(sc, sh_len, pc)) {
            const int tiles = pc.kt1 - pc.kt0, valid = pc.keys - (pc.n_kt - 1) * 128;
            const int gt = g + pc.n_kt - 1 - pc.first;         // when the unit's last key tile comes
            g += tiles;
            if (valid >= 128 || gt >= g) continue;
            const int pi = gt % A::PAIRS, slot = (2 * gt + 1) % A::SLOTS;
            ok = mbar_wait(&v_tail[pi], ph >> pi & 1u, err, ERR_WAIT_PRODUCER);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ph ^= 1u << pi;
            // rows are 128 bytes in each region whatever the swizzle of their 16-byte pieces
            for (int r = 0; r < A::NR; ++r)
                for (int x = max(valid, 0) * 8 + lane; x < 128 * 8; x += 32)
                    *reinterpret_cast<uint4 *>(sKV + slot * A::KV_BYTES + r * A::REGION + x * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&pair[pi]);
        }
    } else if (warp >= A::W_MMA) {
        // ------------------------------------------------------ MMA issue
        // The warp runs converged; one elected lane issues each instruction.
        constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false);
        constexpr uint32_t idesc_o = idesc_bf16(128, HD, false, true);
        const uint64_t dQ0 = sdesc_sw128(smem_u32(sQ), 16, 1024);
        const uint64_t dK0 = sdesc_sw128(smem_u32(sKV), 16, 1024);
        const uint64_t dV0 = sdesc_sw128(smem_u32(sKV), A::REGION, 1024);
        // (issued for both tiles also where a unit has rows in the first only: a
        // branch around the instructions cost 3 % on the large shapes)
        auto issue_s = [&](int i, int slot) {          // S_i = Q_i K^T
            const uint64_t dq = dQ0 + (uint64_t)((i * A::Q_BYTES) >> 4);
            const uint64_t dk = dK0 + (uint64_t)((slot * A::KV_BYTES) >> 4);
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                const uint32_t off = ((ks >> 2) * A::REGION + (ks & 3) * 32) >> 4;
                tc_mma_warp(tmem + A::S_COL(i), dq + off, dk + off, idesc_s, ks > 0 ? 1u : 0u);
            }
            tc_commit_warp(&s_full[i]);
        };
        auto issue_pv = [&](int i, int slot, bool fresh, int half) {   // O_i (+)= P_i V over 64 keys, P_i in TMEM
            const uint64_t dv = dV0 + (uint64_t)((slot * A::KV_BYTES) >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int ks = 4 * half + k;
                tc_mma_tmem_a_warp(tmem + A::O_COL(i), tmem + A::P_COL(i) + 8 * ks, dv + ((ks * 16 * 128) >> 4), idesc_o,
                                   (!fresh || ks > 0) ? 1u : 0u);
            }
        };
        auto wait = [&](uint64_t *b, int parity) -> bool {
            if (__all_sync(0xffffffffu, mbar_try_wait(smem_u32(b), parity & 1))) return true;
            const bool r = mbar_wait(b, parity & 1, err, ERR_WAIT_MMA);
            return __all_sync(0xffffffffu, r) != 0;
        };
        // S runs one key tile ahead of P V.  A look at a barrier that has long
        // completed costs 150 cycles and more next to the busy softmax warps,
        // in which nothing is issued, so there are few: V_g and K_g+1 share one, the queries' and the output's only stand at
        // a piece's first tile (12 heads x 128, 2 x 4320 queries, 30240 keys:
        // 3000 cycles a key tile with separate ones and a tile cursor).
        bool ok = walk.next(sc, sh_len, pc) && wait(q_full, 0) && wait(k0_full, 0);
        const int i_own = warp - A::W_MMA;                 // SEP_P: the row tile of this warp
        int g = 0, p = 0, left = pc.kt1 - pc.kt0;          // left: key tiles of the piece from g on
        bool fresh = true;                                 // g is the piece's first
        int sk = 0, sv = 1;                                // slots of K_g+1 and V_g
        auto two_on = [&](int s) { return s + 2 >= A::SLOTS ? s + 2 - A::SLOTS : s + 2; };
        if (ok) {
            tc_fence_after();
            issue_s(A::SEP_P ? i_own : 0, 0);
            if constexpr (!A::SEP_P) issue_s(1, 0);
            tc_commit_warp(&empty[0]);
            if (left == 1) tc_commit_warp(q_empty);
        }
        while (ok) {
            sk = two_on(sk);
            const bool last = left == 1;
            bool more = true;
            if (last) {
                more = walk.next(sc, sh_len, pc);
                left = more ? pc.kt1 - pc.kt0 : 0;
                if (A::SEP_P && more && !wait(q_full, p + 1)) break;
            } else {
                --left;
            }
            if (!wait(&pair[g % A::PAIRS], g / A::PAIRS)) break;
            if constexpr (A::SEP_P) {
                // S_i of the next tile as soon as the softmax has read S_i, then
                // P_i V, its first half while the softmax is at the second
                const int i = i_own;
                if (more) {
                    if (!wait(&s_cons[i], g)) break;
                    tc_fence_after();
                    issue_s(i, sk);
                    tc_commit_warp(&empty[sk]);
                    if (left == 1) tc_commit_warp(q_empty);
                }
                if (fresh && p > 0 && !wait(&o_free[i], p - 1)) break;
                if (!wait(&p_half[i], g)) break;
                tc_fence_after();
                issue_pv(i, sv, fresh, 0);
                if (!wait(&p_full[i], g)) break;
                tc_fence_after();
                issue_pv(i, sv, fresh, 1);
                tc_commit_warp(&pv_done[i]);
                tc_commit_warp(&empty[sv]);
            } else {
                // P_i overwrites S_i: P0 V, next S0, P1 V, next S1 -- the order
                // in which the warpgroups finish (the next piece's queries, on
                // their way, hold up its S0 only)
                if (fresh && p > 0 && !wait(&o_free[0], p - 1)) break;
                if (!wait(&p_full[0], g)) break;
                tc_fence_after();
                issue_pv(0, sv, fresh, 0);
                issue_pv(0, sv, fresh, 1);
                if (last) tc_commit_warp(&pv_done[0]);
                if (last && more && !wait(q_full, p + 1)) break;
                if (more) issue_s(0, sk);
                if (fresh && p > 0 && !wait(&o_free[1], p - 1)) break;
                if (!wait(&p_full[1], g)) break;
                tc_fence_after();
                issue_pv(1, sv, fresh, 0);
                issue_pv(1, sv, fresh, 1);
                tc_commit_warp(&empty[sv]);
                if (last) tc_commit_warp(&pv_done[1]);
                if (more) {
                    issue_s(1, sk);
                    tc_commit_warp(&empty[sk]);
                    if (left == 1) tc_commit_warp(q_empty);
                }
            }
            if (!more) break;
            sv = two_on(sv);
            fresh = last;
            p += last ? 1 : 0;
            ++g;
        }
    } else {
        // ------------------------------------------------------------ softmax
        const int wg = warp >> 2, q = warp & 3;
        const int r = q * 32 + lane;                       // row of the 128-row tile
        const int tl_ = wg * tt1 + r / sc.grp, gq = r - (r / sc.grp) * sc.grp;   // token of the unit, head of the group
        const bool in_tile = r < tt1 * sc.grp;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t tS = lanes + A::S_COL(wg), tP = lanes + A::P_COL(wg), tO = lanes + A::O_COL(wg);
        // One key tile: S_i -> running max m, P_i = 2^(S_i sl2 - m) into TMEM,
        // running sum l.  cols: keys of this tile the row sees; masked: some
        // row of the warp does not see all 128.  false: a wait ran out.
        auto tile = [&](int g, int cols, bool masked, bool fresh, float &m, float &l) -> bool {
            bool ok = mbar_wait(&s_full[wg], g & 1, err, ERR_WAIT_SOFTMAX);
            __syncwarp();
            if (!__all_sync(0xffffffffu, ok)) return false;
            tc_fence_after();
            float s[128];
            tmem_ld128_sync(tS, s);
            if constexpr (A::SEP_P) {
                tc_fence_before();
                mbar_arrive(&s_cons[wg]);
            }
            if (masked) {
#pragma unroll
                for (int c = 0; c < 128; ++c)
                    if (c >= cols) s[c] = -INFINITY;
            }
            float mx[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) mx[k] = s[k];
#pragma unroll
            for (int c = 16; c < 112; c += 32) {
#pragma unroll
                for (int k = 0; k < 16; ++k) mx[k] = max3(mx[k], s[c + k], s[c + 16 + k]);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) mx[k] = fmaxf(mx[k], s[112 + k]);
#pragma unroll
            for (int k = 0; k < 5; ++k) mx[k] = max3(mx[k], mx[k + 5], mx[k + 10]);
            const float m_new = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[15]), mx[0]) * sl2;
            // a row that has seen no key yet: m = -inf, every weight 0; its first
            // key scales the (zero) sums by 2^-inf = 0
            if (fresh) m = m_new;
            const bool grow = !fresh && m_new > m + A::LAZY;
            const float alpha = grow ? exp2_mufu(m - m_new) : 1.0f;
            if (grow) m = m_new;
            if constexpr (A::SEP_P) {
                // P_i free and O_i stable once P V of the previous tile is done
                if (g >= 1) {
                    ok = mbar_wait(&pv_done[wg], (g - 1) & 1, err, ERR_WAIT_SOFTMAX);
                    __syncwarp();
                    if (!__all_sync(0xffffffffu, ok)) return false;
                    tc_fence_after();
                }
            }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll 1
                for (int c = 0; c < HD / 16; ++c) {
                    float t[16];
                    tmem_ld16_sync(tO + 16 * c, t);
#pragma unroll
                    for (int i = 0; i < 16; ++i) t[i] *= alpha;
                    tmem_st16_sync(tO + 16 * c, t);
                }
            }
            if constexpr (A::TURNS) {
                // the two warps of an SM sub-partition take turns on the
                // MUFU-bound exponentials
                if (wg == 1 || g > 0) {
                    ok = mbar_wait(&turn[4 * wg + q], (wg == 1 ? g : g - 1) & 1, err, ERR_WAIT_SOFTMAX);
                    __syncwarp();
                    if (!__all_sync(0xffffffffu, ok)) return false;
                }
            }
            const float nm = m == -INFINITY ? 0.0f : -m;
            const float2 sc2 = make_float2(sl2, sl2), nm2 = make_float2(nm, nm);
            float2 rs0 = make_float2(0.f, 0.f), rs1 = make_float2(0.f, 0.f);
#pragma unroll
            for (int qt = 0; qt < 4; ++qt) {
                uint32_t w[16];
#pragma unroll
                for (int k = 0; k < 16; k += 2) {
                    const int c = 32 * qt + 2 * k;
                    const float2 a = __ffma2_rn(make_float2(s[c], s[c + 1]), sc2, nm2);
                    const float2 b = __ffma2_rn(make_float2(s[c + 2], s[c + 3]), sc2, nm2);
                    const float2 pa = make_float2(exp2_mufu(a.x), exp2_mufu(a.y));
                    const float2 pb = make_float2(exp2_mufu(b.x), exp2_mufu(b.y));
                    rs0 = __fadd2_rn(rs0, pa);
                    rs1 = __fadd2_rn(rs1, pb);
                    const __nv_bfloat162 h0 = __floats2bfloat162_rn(pa.x, pa.y);
                    const __nv_bfloat162 h1 = __floats2bfloat162_rn(pb.x, pb.y);
                    w[k] = *reinterpret_cast<const uint32_t *>(&h0);
                    w[k + 1] = *reinterpret_cast<const uint32_t *>(&h1);
                }
                tmem_st16u_sync(tP + 16 * qt, w);
                if (A::SEP_P && qt == 1) {
                    tc_fence_before();
                    mbar_arrive(&p_half[wg]);
                }
            }
            const float2 rs = __fadd2_rn(rs0, rs1);
            l = l * alpha + (rs.x + rs.y);
            tc_fence_before();
            mbar_arrive(&p_full[wg]);
            __syncwarp();
            if constexpr (A::TURNS)
                if (lane == 0) mbar_arrive(&turn[4 * (wg ^ 1) + q]);
            return true;
        };
        // The same steps of a warp none of whose rows exist: barriers only.
        auto idle_tile = [&](int g) -> bool {
            bool ok = mbar_wait(&s_full[wg], g & 1, err, ERR_WAIT_SOFTMAX);
            if constexpr (A::SEP_P) {
                mbar_arrive(&s_cons[wg]);
                if (g >= 1) ok = ok && mbar_wait(&pv_done[wg], (g - 1) & 1, err, ERR_WAIT_SOFTMAX);
            }
            if constexpr (A::TURNS)
                if (wg == 1 || g > 0)
                    ok = ok && mbar_wait(&turn[4 * wg + q], (wg == 1 ? g : g - 1) & 1, err, ERR_WAIT_SOFTMAX);
            ok = __all_sync(0xffffffffu, ok);
            if constexpr (A::SEP_P) mbar_arrive(&p_half[wg]);
            mbar_arrive(&p_full[wg]);
            if constexpr (A::TURNS)
                if (lane == 0) mbar_arrive(&turn[4 * (wg ^ 1) + q]);
            return ok;
        };
        // The walk of a softmax warp lives in shared memory, so that its piece
        // takes no registers during the key tiles.
        BranchWarpWalk &ww = sh_walk[warp];
        auto advance = [&](int slot) {
            __syncwarp();
            if (lane == 0) {
                BranchWalk<128> w = ww.w;
                BranchPiece c;
                ww.more = w.next(sc, sh_len, c);
                ww.w = w;
                ww.pc[slot] = c;
            }
            __syncwarp();
        };
        if (lane == 0) ww.w = walk;
        advance(0);
        int g = 0, p = 0;
        bool ok = true;
        while (ok && ww.more) {
            const BranchPiece &cur = ww.pc[p & 1];
            const bool row_ok = in_tile && tl_ < cur.nt;
            const bool live = __any_sync(0xffffffffu, row_ok) != 0;
            int see = 1 << 30;                             // keys of the unit this row sees
            if (row_ok) {
                const int t = cur.t0 + tl_, b = cur.idx < sc.n_pr ? t / sc.n_q : cur.b;
                see = min(sc.limit(sc.seq_len(b, sh_len), t - b * sc.n_q) - cur.key0, cur.keys);
            }
            float m = -INFINITY, l = 0.0f;
            const int g_end = g + cur.kt1 - cur.kt0, wrap = cur.n_kt * 128;
            bool fresh = true;
            if (live) {
                const int least = __reduce_min_sync(0xffffffffu, see);
                for (int key = cur.first * 128; g < g_end; ++g) {
                    ok = tile(g, see - key, least < key + 128, fresh, m, l);
                    if (!ok) break;
                    fresh = false;
                    key = key + 128 == wrap ? 0 : key + 128;
                }
            } else {
                for (; ok && g < g_end; ++g) ok = idle_tile(g);
            }
            if (!ok) break;
            advance((p + 1) & 1);                          // while the last P V runs
            ok = mbar_wait(&pv_done[wg], (A::SEP_P ? g - 1 : p) & 1, err, ERR_WAIT_SOFTMAX);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (!live) {
                tc_fence_before();
                mbar_arrive(&o_free[wg]);
                ++p;
                continue;
            }
            float x[HD];
            if constexpr (HD == 128) {
                tmem_ld128_sync(tO, x);
            } else {
                tmem_ld32_sync(tO, *reinterpret_cast<float(*)[32]>(x));
                tmem_ld32_sync(tO + 32, *reinterpret_cast<float(*)[32]>(x + 32));
            }
            tc_fence_before();
            mbar_arrive(&o_free[wg]);                      // the next piece may write O_i
            const BranchPiece c = cur;
            if (sc.n_pr == 0 && c.kt1 - c.kt0 == c.n_kt) {
                if (sc.lse != nullptr && row_ok) sc.put_lse(c.t0 + tl_, c.h * sc.grp + gq, m, l);
                // Whole unit: 32 columns (64 bytes) of a row at a time.  Each
                // quad of lanes exchanges its four rows' 16-byte parts, so
                // that a store covers 64 consecutive bytes of 8 rows.
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                const long long mine = row_ok ? (long long)(c.t0 + tl_) * o_ld + (c.h * sc.grp + gq) * HD : -1;
                long long at[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) at[j] = __shfl_sync(0xffffffffu, mine, (lane & ~3) + j);
#pragma unroll
                for (int cb = 0; cb < HD / 32; ++cb) {
                    uint4 u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int at_c = 32 * cb + 8 * i + 2 * j;
                            const __nv_bfloat162 y = __floats2bfloat162_rn(x[at_c] * inv, x[at_c + 1] * inv);
                            w[j] = *reinterpret_cast<const uint32_t *>(&y);
                        }
                        u[i] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    quad_transpose(u, lane);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at[j] >= 0) *reinterpret_cast<uint4 *>(o + at[j] + 32 * cb + 8 * (lane & 3)) = u[j];
                }
            } else if (row_ok) {
                const long row0 = branch_slot_row(sc, c, blockIdx.x, p == 0);
                const int rr = tl_ * sc.grp + gq, pitch = c.idx < sc.n_pr ? sc.pitch_p : sc.pitch_o;
                float4 *dst = reinterpret_cast<float4 *>(sc.ws_o + row0 * HD) + rr;
#pragma unroll
                for (int i = 0; i < HD / 4; ++i)
                    dst[(size_t)i * pitch] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                sc.ws_ml[row0 + rr] = make_float2(m, l);
            }
            ++p;
        }
    }
    pdl_release();
    tc_fence_before();
    __syncthreads();
    if (warp == A::W_MMA) {
        tc_fence_after();
        tmem_dealloc(tmem, A::TMEM_COLS);
    }
}

// ------------------------------------------------------------ fp32 kernel
// 64-row x 64-key tiles, 256 threads as 16 x 16: thread (ty, tx) computes
// scores of rows 4 ty.. and keys tx + 16 j, and of the same rows' output one or
// two groups of four columns, over one of KS interleaved shares of the keys
// where a row has fewer than 16 groups (the shares meet at a piece's end): 12
// shared-memory accesses per 64 FMAs in either product.  The next tile's keys
// and values come by asynchronous copies.  exp2f, no bf16 anywhere.  8 heads, 4
// x 512 causal queries over 4096 + 512..1024 keys: 171 / 507 / 1031 us at head
// size 16 / 64 / 128, 28 / 38 / 37.5 TFLOP/s of about 80: the shared-memory
// pipe is 64 / 77 / 68 % and the issue slots 71 / 71 / 63 % busy, the FMA pipe 48
// / 56 / 52 %.  Short calls are a few tiles a CTA: 4 x 232 tokens, 4 heads x 16,
// 696 keys 19.4 us.
// CTAs an SM where a call has work for them (what fits in shared memory): 2
// against 1 take 171 / 203 and 507 / 591 us above, but 18.6 / 15.7 us where 2 x
// 77 queries over some 380 keys leave a CTA one tile or none.
constexpr int branch_f32_ctas(int hd) { return hd <= 64 ? 2 : 1; }
template <int HD>
struct BranchTileF32 {
    static constexpr int RT = 64, KT = 64, LD = HD + 4, LDP = KT + 4;
    static constexpr int SMEM_BYTES = (5 * 64 * LD + 64 * LDP) * (int)sizeof(float);
    static constexpr int CG = HD / 4 < 16 ? HD / 4 : 16;   // column groups side by side
    static constexpr int KS = 16 / CG, NV = HD / (4 * CG); // shares of the keys, column groups of a thread
    static constexpr int CTAS = branch_f32_ctas(HD);       // resident on an SM
};
// 16 bytes to shared memory, of which `bytes` are read and the rest are zero
__device__ __forceinline__ void cp_async16(uint32_t dst, const float *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int HD>
__global__ void __launch_bounds__(256, BranchTileF32<HD>::CTAS)
    branch_attn_f32_kernel(const float *q, const long q_ld, const float *__restrict__ k, const float *__restrict__ v,
                           float *o, const long o_ld, const float sl2, const __grid_constant__ BranchSched sc, int *err) {
    using A = BranchTileF32<HD>;
    pdl_wait();
    extern __shared__ __align__(16) float sm[];
    __shared__ int sh_len[2 * LEN_CACHE], sh_scan[16];
    __shared__ BranchStart sh_start;
    const BranchStart start = branch_start<64>(sc, sh_len, sh_scan, &sh_start);
    branch_zero_rows<float>(sc, sh_len, o, o_ld, sc.Hk * sc.grp * HD);
    if (blockIdx.x == 0 && threadIdx.x < 32) branch_publish<64>(sc, sh_len, err);
    float *sQ = sm, *sKV = sQ + 64 * A::LD, *sP = sKV + 4 * 64 * A::LD;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int log_ps = 31 - __clz(sc.ps);
    const size_t ld = (size_t)sc.Hk * HD;
    constexpr int V4 = HD / 4;                             // float4 of a row
    constexpr int NC = HD / 16;                            // float4 of K and of V that a thread loads
    const int cg = tx % A::CG, ks = tx / A::CG;
    BranchWalk<64> walk(sc, start);
    BranchPiece pc;
    int np = 0;
    while (walk.next(sc, sh_len, pc)) {
        const int rows = pc.nt * sc.grp, row_id = sc.table_row(pc.b, sh_len);
        __syncthreads();
        for (int x = tid; x < 64 * V4; x += 256) {
            const int r = x / V4, c = x % V4;
            float4 f = make_float4(0, 0, 0, 0);
            if (r < rows)
                f = *reinterpret_cast<const float4 *>(q + (size_t)(pc.t0 + r / sc.grp) * q_ld +
                                                      (pc.h * sc.grp + r % sc.grp) * HD + 4 * c);
            *reinterpret_cast<float4 *>(sQ + r * A::LD + 4 * c) = f;
        }
        int see[4];
        float m[4], l[4];                                  // l: of this thread's keys
        float4 acc[4][A::NV];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i;
            see[i] = 0;
            if (r < rows) {
                const int t = pc.t0 + r / sc.grp, b = t / sc.n_q;
                see[i] = min(sc.limit(sc.seq_len(b, sh_len), t - b * sc.n_q) - pc.key0, pc.keys);
            }
            m[i] = -INFINITY;
            l[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < A::NV; ++j) acc[i][j] = make_float4(0, 0, 0, 0);
        }
        // the next tile's rows are on their way while this one is at work
        auto fetch = [&](int kt) {
            float *dst = sKV + ((kt - pc.kt0) & 1) * (2 * 64 * A::LD);
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int x = tid + 256 * i, r = x / V4, c = x % V4, key = kt * 64 + r;
                size_t off = 0;
                int bytes = 0;                             // 0: the row is filled with zeros
                if (key < pc.keys && row_id >= 0) {
                    const int at = pc.key0 + key;
                    const int id = sc.table[(size_t)row_id * sc.max_pages + (at >> log_ps)];
                    if (id >= 0 && id < sc.n_pages) {
                        off = ((size_t)id * sc.ps + (at & (sc.ps - 1))) * ld + pc.h * HD + 4 * c;
                        bytes = 16;
                    } else if (err) {
                        atomicOr(err, ERR_BAD_SEQ);
                    }
                }
                cp_async16(smem_u32(dst + r * A::LD + 4 * c), k + off, bytes);
                cp_async16(smem_u32(dst + (64 + r) * A::LD + 4 * c), v + off, bytes);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        fetch(pc.kt0);
        for (int kt = pc.kt0; kt < pc.kt1; ++kt) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();
            if (kt + 1 < pc.kt1) fetch(kt + 1);
            const float *sK = sKV + ((kt - pc.kt0) & 1) * (2 * 64 * A::LD), *sV = sK + 64 * A::LD;
            if (4 * (ty & ~1) < rows) {                    // the warp (thread rows 2 w, 2 w + 1) has rows
                float s[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
#pragma unroll 4
                for (int c = 0; c < HD; c += 4) {
                    float4 a[4], b[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4 *>(sQ + (4 * ty + i) * A::LD + c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4 *>(sK + (tx + 16 * j) * A::LD + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[i][j] = fmaf(a[i].x, b[j].x, s[i][j]);
                            s[i][j] = fmaf(a[i].y, b[j].y, s[i][j]);
                            s[i][j] = fmaf(a[i].z, b[j].z, s[i][j]);
                            s[i][j] = fmaf(a[i].w, b[j].w, s[i][j]);
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = kt * 64 + tx + 16 * j < see[i] ? s[i][j] * sl2 : -INFINITY;
                        mx = fmaxf(mx, s[i][j]);
                    }
#pragma unroll
                    for (int d = 8; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    const float mn = fmaxf(m[i], mx), use = mn == -INFINITY ? 0.0f : mn;
                    const float alpha = exp2f(m[i] - use);
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float pj = exp2f(s[i][j] - use);
                        sum += pj;
                        sP[(4 * ty + i) * A::LDP + tx + 16 * j] = pj;
                    }
                    l[i] = l[i] * alpha + sum;
                    m[i] = mn;
#pragma unroll
                    for (int j = 0; j < A::NV; ++j) {
                        acc[i][j].x *= alpha;
                        acc[i][j].y *= alpha;
                        acc[i][j].z *= alpha;
                        acc[i][j].w *= alpha;
                    }
                }
                __syncwarp();                              // a warp reads only its own rows of P
#pragma unroll 2
                for (int c = 4 * ks; c < 64; c += 4 * A::KS) {
                    float pr[4][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4 *>(pr[i]) = *reinterpret_cast<const float4 *>(sP + (4 * ty + i) * A::LDP + c);
#pragma unroll
                    for (int j = 0; j < A::NV; ++j)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float4 b = *reinterpret_cast<const float4 *>(sV + (c + x) * A::LD + 4 * (cg + A::CG * j));
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                acc[i][j].x = fmaf(pr[i][x], b.x, acc[i][j].x);
                                acc[i][j].y = fmaf(pr[i][x], b.y, acc[i][j].y);
                                acc[i][j].z = fmaf(pr[i][x], b.z, acc[i][j].z);
                                acc[i][j].w = fmaf(pr[i][x], b.w, acc[i][j].w);
                            }
                        }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
#pragma unroll
            for (int d = 8; d >= A::CG; d >>= 1)
#pragma unroll
                for (int j = 0; j < A::NV; ++j) {
                    acc[i][j].x += __shfl_xor_sync(0xffffffffu, acc[i][j].x, d);
                    acc[i][j].y += __shfl_xor_sync(0xffffffffu, acc[i][j].y, d);
                    acc[i][j].z += __shfl_xor_sync(0xffffffffu, acc[i][j].z, d);
                    acc[i][j].w += __shfl_xor_sync(0xffffffffu, acc[i][j].w, d);
                }
        }
        const bool whole = sc.n_pr == 0 && pc.kt1 - pc.kt0 == pc.n_kt;
        const long row0 = whole ? 0 : branch_slot_row(sc, pc, blockIdx.x, np == 0);
        const int pitch = pc.idx < sc.n_pr ? sc.pitch_p : sc.pitch_o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i;
            if (r >= rows) continue;
            const bool mine = i % A::KS == ks;             // every share holds the sums: row by row another writes
            if (whole) {
                const float inv = l[i] > 0.0f ? 1.0f / l[i] : 0.0f;
                if (sc.lse != nullptr && tx == 0) sc.put_lse(pc.t0 + r / sc.grp, pc.h * sc.grp + r % sc.grp, m[i], l[i]);
                float *dst = o + (size_t)(pc.t0 + r / sc.grp) * o_ld + (pc.h * sc.grp + r % sc.grp) * HD;
#pragma unroll
                for (int j = 0; j < A::NV; ++j)
                    if (mine)
                        *reinterpret_cast<float4 *>(dst + 4 * (cg + A::CG * j)) =
                            make_float4(acc[i][j].x * inv, acc[i][j].y * inv, acc[i][j].z * inv, acc[i][j].w * inv);
            } else {
#pragma unroll
                for (int j = 0; j < A::NV; ++j)
                    if (mine)
                        *reinterpret_cast<float4 *>(sc.ws_o + row0 * HD + ((size_t)(cg + A::CG * j) * pitch + r) * 4) = acc[i][j];
                if (tx == 0) sc.ws_ml[row0 + r] = make_float2(m[i], l[i]);
            }
        }
        ++np;
    }
}

// ---------------------------------------------------------------- combine
// Adds the pieces of a row's prefix unit and of its own unit in CTA order.
// PREFIX: grid.x is (key head, own entry), and every row is merged.  Else
// grid.x is the CTA boundaries, of which the first one inside a unit merges
// it (units that one CTA ran whole are written already).  grid.y: NI RB rows
// of the unit.  A thread owns four columns of a row, neighbouring threads
// neighbouring rows.  Latency bound, so the loads of NI rows x KB pieces are
// in flight together: 4 rows and 2 pieces where few pieces meet many rows;
// with PREFIX one row and 8 pieces, or 4 with more CTAs resident where a row
// has few, and the row slots that a short tile leaves idle take a share of the
// pieces each (their sums meet in shared memory, in a fixed order).  Measured: 7
// us after the last piece of 32 single tokens (19 pieces a row), 9 for 16 branches
// of 20 tokens, 13.6 for 6 prompts of 1031 (cut units of 252 rows).
constexpr int COMBINE_THREADS = 256, COMBINE_SMALL = 64;
template <typename T, int HD, bool PREFIX, int THREADS, int KB>
__global__ void __launch_bounds__(THREADS, PREFIX ? (KB == 8 ? 3 : 4) * COMBINE_THREADS / THREADS : 0)
    branch_combine_kernel(T *o, const long o_ld, const __grid_constant__ BranchSched s) {
    pdl_wait();
    constexpr int RB = THREADS / (HD / 4), NI = PREFIX ? 1 : 4;
    const unsigned PP = PREFIX ? (unsigned)s.n_pr * s.line_len(s.n_pt) : 0;
    int h, e, off, len;                                    // own unit: position in its head's line, line length
    if (PREFIX) {
        h = blockIdx.x / s.E;
        e = blockIdx.x - h * s.E;
        off = s.ws_off[e];
        len = s.ws_off[e + 1] - off;
    } else {
        const int4 st = s.ws_start[blockIdx.x + 1];
        h = st.x;
        e = st.y;
        off = st.z;
        len = s.line_len(st.w);
    }
    const unsigned Th = PP + s.ws_off[s.E], Tl = Th * s.Hk;
    const BranchLine line(Tl, s.G);
    unsigned so;                                           // the own unit's start on the line
    int no = 0, co = 0;                                    // its pieces, their first CTA
    if (PREFIX) {
        so = h * Th + PP + off;
        if (len > 0) {
            co = line.owner(so + s.lead);
            no = line.owner(so + len - 1) - co + 1;
        }
    } else {
        const unsigned c = blockIdx.x + 1, x = line.begin(c);
        if (x >= Tl || off <= s.lead) return;          // no key tile of the unit lies before CTA c
        so = x - off;
        co = c - 1;
        if (line.begin(co) > so + s.lead) return;      // an earlier boundary merges the unit
        no = line.owner(so + len - 1) - co + 1;
    }
    const int b = e / s.n_st, i0 = (e - b * s.n_st) * s.tt;
    const int rows = min(s.tt, s.n_q - i0) * s.grp;
    const int ch = threadIdx.x / RB, slot_r = threadIdx.x % RB, first_row = blockIdx.y * (NI * RB);
    if (first_row >= rows) return;
    // PREFIX: 2^lg row slots hold the rows that are left, the others shares of the pieces
    int lg = 0;
    if (PREFIX)
        while ((1 << lg) < RB && (1 << lg) < rows - first_row) ++lg;
    const int share = PREFIX ? slot_r >> lg : 0, n_share = PREFIX ? RB >> lg : 1;
    const int r0 = first_row + (PREFIX ? slot_r & ((1 << lg) - 1) : slot_r);
    const bool there = r0 < rows;
    if (!PREFIX && !there) return;
    int np = 0;
    const float4 *px = nullptr;                            // first prefix piece: this row's float4, (m, l)
    const float2 *pml = nullptr;
    if (PREFIX) {
        const int rr = min(r0, rows - 1), t = b * s.n_q + i0 + rr / s.grp, pi = t / s.tt;
        const int in = (t - pi * s.tt) * s.grp + rr % s.grp;
        const unsigned s0 = h * Th + (unsigned)pi * s.line_len(s.n_pt) + s.lead;
        const int cp = line.owner(s0);
        np = line.owner(s0 + s.n_pt - 1) - cp + 1;
        const long slot = ((long)h * s.n_pr + pi + cp) * s.pitch_p;
        px = reinterpret_cast<const float4 *>(s.ws_o + slot * HD) + (size_t)ch * s.pitch_p + in;
        pml = s.ws_ml + slot + in;
    }
    const long own0 = s.slots_p * s.pitch_p + ((long)h * s.E + e + co) * s.pitch_o;
    const int n = np + no;
    float m[NI], den[NI];
    float4 acc[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        m[i] = -INFINITY;
        den[i] = 0.0f;
        acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 1
    for (int k0 = share; k0 < n; k0 += KB * n_share) {
        float4 x[NI][KB];
        float2 ml[NI][KB];
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            const int at = k0 + k * n_share, kk = min(at, n - 1);   // a piece that exists: its loads are always sound
            const bool pre = PREFIX && kk < np;
            long slot = 0;                                 // the own slot's first row
            if (!pre) slot = PREFIX ? own0 + (long)(kk - np) * s.pitch_o : (2l * (co + kk) + (line.begin(co + kk) >= so ? 0 : 1)) * s.pitch_o;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int r = min(r0 + i * RB, rows - 1);
                x[i][k] = pre ? px[(size_t)kk * s.pitch_p * (HD / 4)]
                              : reinterpret_cast<const float4 *>(s.ws_o + slot * HD)[(size_t)ch * s.pitch_o + r];
                ml[i][k] = pre ? pml[(size_t)kk * s.pitch_p] : s.ws_ml[slot + r];
                if (at >= n) ml[i][k] = make_float2(-INFINITY, 0.0f);
            }
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            float top = m[i];
#pragma unroll
            for (int k = 0; k < KB; ++k) top = fmaxf(top, ml[i][k].x);
            const float use = top == -INFINITY ? 0.0f : top;
            const float a = exp2f(m[i] - use);
            m[i] = top;
            den[i] *= a;
            acc[i] = make_float4(acc[i].x * a, acc[i].y * a, acc[i].z * a, acc[i].w * a);
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                // no key of this piece for the row; a row of NaN has no maximum either, but a sum that is NaN
                if (ml[i][k].x == -INFINITY && ml[i][k].y == 0.0f) continue;
                const float w = exp2f(ml[i][k].x - use);
                den[i] = fmaf(w, ml[i][k].y, den[i]);
                acc[i].x = fmaf(w, x[i][k].x, acc[i].x);
                acc[i].y = fmaf(w, x[i][k].y, acc[i].y);
                acc[i].z = fmaf(w, x[i][k].z, acc[i].z);
                acc[i].w = fmaf(w, x[i][k].w, acc[i].w);
            }
        }
    }
    if constexpr (PREFIX) {
        __shared__ float4 sh_x[THREADS];
        __shared__ float2 sh_ml[THREADS];
        if (n_share > 1) {
            sh_x[threadIdx.x] = acc[0];
            sh_ml[threadIdx.x] = make_float2(m[0], den[0]);
            __syncthreads();
            if (share > 0) return;
            float top = m[0];
            for (int j = 1; j < n_share; ++j) top = fmaxf(top, sh_ml[threadIdx.x + (j << lg)].x);
            const float use = top == -INFINITY ? 0.0f : top;
            m[0] = top;
            den[0] = 0.0f;
            acc[0] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int j = 0; j < n_share; ++j) {
                const float2 ml = sh_ml[threadIdx.x + (j << lg)];
                const float4 x = sh_x[threadIdx.x + (j << lg)];
                const float w = exp2f(ml.x - use);         // 0 for a share without keys, whose sums are 0
                den[0] = fmaf(w, ml.y, den[0]);
                acc[0].x = fmaf(w, x.x, acc[0].x);
                acc[0].y = fmaf(w, x.y, acc[0].y);
                acc[0].z = fmaf(w, x.z, acc[0].z);
                acc[0].w = fmaf(w, x.w, acc[0].w);
            }
        }
        if (!there) return;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = r0 + i * RB;
        if (r >= rows) break;
        const float inv = den[i] > 0.0f ? 1.0f / den[i] : 0.0f;
        const int tr = r / s.grp;
        if (s.lse != nullptr && ch == 0) s.put_lse(b * s.n_q + i0 + tr, h * s.grp + r - tr * s.grp, m[i], den[i]);
        T *dst = o + (size_t)(b * s.n_q + i0 + tr) * o_ld + (h * s.grp + r - tr * s.grp) * HD + 4 * ch;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(dst) = make_float4(acc[i].x * inv, acc[i].y * inv, acc[i].z * inv, acc[i].w * inv);
        } else {
            const __nv_bfloat162 y0 = __floats2bfloat162_rn(acc[i].x * inv, acc[i].y * inv);
            const __nv_bfloat162 y1 = __floats2bfloat162_rn(acc[i].z * inv, acc[i].w * inv);
            *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&y0), *reinterpret_cast<const uint32_t *>(&y1));
        }
    }
}

// ------------------------------------------------------------------- host
struct BranchPlan {
    BranchSched s;
    int qt, tt1;
    size_t rows, bytes;       // partial rows, workspace bytes
};
static BranchPlan branch_plan(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    BranchPlan p;
    BranchSched &s = p.s;
    s = BranchSched{};
    const bool f32 = c.dtype == XC_F32;
    const int RT = f32 ? 64 : 128, KT = f32 ? 64 : 128;
    s.B = B;
    s.n_q = n_q;
    s.Hk = c.n_kv_heads;
    s.grp = H / s.Hk;
    s.ps = c.page_size;
    s.max_seqs = c.max_seqs;
    s.max_pages = c.max_pages;
    s.n_pages = c.n_pages;
    s.len = c.len;
    s.table = c.table;
    s.G = device_sms();
    p.tt1 = RT / s.grp;
    // Prefix units where the tiles saved by packing the branches' rows (the shared
    // keys of every entry) outweigh what they bring: a lead each, and partials,
    // where whole units write their output: about two key tiles for the rows of
    // a prefix tile and as much, by the rows it has, for an entry.  With them and
    // without, 46 branches of 440 tokens over 864 shared keys, 16 / 8 heads x 128:
    // 565 and 229 us; 16 branches of 20 tokens over 12960: 51 and 154; 200 single
    // tokens over 256, 32 / 8 heads x 128: 63 and 97.
    // Two row tiles per CTA where that makes the shorter line: a key tile of one
    // counts 2 against 3, a branch's own keys (the host does not know them) as one
    // key tile and its new tokens.  One against two tiles: 200 single tokens over
    // 256 + 16..120 keys, 32 / 8 heads x 64 48 and 58 us, 16 branches of 20 tokens
    // over 12960 keys 50.8 and 52.9; but 32 single tokens over 38880 + 1..1500
    // keys, 40 / 8 heads x 128 76.6 and 63.4, 6 prompts of 1031 tokens 70.7 and 65.9.
    const long long tokens = (long long)B * n_q, n_pt = (shared + KT - 1) / KT, own = 1 + n_q / KT;
    long long least = 0;
    for (int qt = 1; qt <= (f32 ? 1 : 2); ++qt) {
        const int tt = p.tt1 * qt, n_st = (n_q + tt - 1) / tt;
        const long long E = (long long)B * n_st, packed = (tokens + tt - 1) / tt;
        const long long rows = std::min(n_q, tt) * s.grp;
        const bool prefix = shared > 0 && E * shared > packed * (n_pt + 4) * KT + 2 * E * rows / qt;
        const long long line = prefix ? packed * (n_pt + 2) + E * (own + 2) : E * (n_pt + own + 2);
        if (qt == 2 && 3 * line >= 2 * least) break;
        least = line;
        p.qt = qt;
        s.tt = tt;
        s.n_st = n_st;
        s.E = (int)E;
        s.P = prefix ? shared : 0;
        s.n_pr = prefix ? (int)packed : 0;
        s.n_pt = prefix ? (int)n_pt : 0;
    }
    // (keys that the host knows of: a CTA on every SM has 8 tiles or more)
    if (f32 && (double)s.E * s.Hk * ((shared + n_q + KT - 1) / KT) >= 8.0 * s.G) s.G *= branch_f32_ctas(c.head_dim);
    // A unit's query load, pipeline ramp and output take about as long as two
    // key tiles (counted 1: 6 prompts of 1031 tokens 71.2 us, counted 2: 65.7; 16
    // branches of 20 tokens over 12960 keys 53.3 and 50.7).
    s.lead = 2;
    s.pitch_p = (int)(tokens < s.tt ? tokens : s.tt) * s.grp;
    s.pitch_o = (n_q < s.tt ? n_q : s.tt) * s.grp;
    s.slots_p = s.n_pr > 0 ? (long)s.Hk * s.n_pr + s.G : 0;
    const size_t slots_o = s.n_pr > 0 ? (size_t)s.Hk * s.E + s.G : 2 * (size_t)s.G;
    p.rows = (size_t)s.slots_p * s.pitch_p + slots_o * s.pitch_o;
    p.bytes = s.G * sizeof(int4) + p.rows * (c.head_dim * sizeof(float) + sizeof(float2)) + ((size_t)s.E + 1) * sizeof(int);
    return p;
}
bool branch_attn_fits(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    const BranchPlan p = branch_plan(c, B, n_q, H, shared);
    const long long kt = c.dtype == XC_F32 ? 64 : 128;
    const long long own = (long long)p.s.E * (((long long)c.max_pages * c.page_size + kt - 1) / kt + p.s.lead);
    return (long long)B * ((n_q + p.s.tt - 1) / p.s.tt) < (1ll << 30) && p.s.Hk * ((long long)p.s.n_pr * (p.s.n_pt + p.s.lead) + own) < (1ll << 31);
}
size_t branch_attn_workspace_bytes(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    return branch_plan(c, B, n_q, H, shared).bytes;
}

template <int HD, int QT>
static cudaError_t launch_tc(const xc_kv_cache &c, const BranchAttnArgs &a, const BranchPlan &p, float sl2, int *err,
                             cudaStream_t st) {
    using A = BranchTile<HD, QT>;
    static DeviceSet asked{0};
    cudaError_t e = allow_smem(branch_attn_kernel<HD, QT>, A::SMEM_BYTES, asked);
    if (e != cudaSuccess) return e;
    const uint64_t rows = (uint64_t)c.n_pages * c.page_size, cols = (uint64_t)c.n_kv_heads * HD;
    const uint32_t box = c.page_size < 128 ? c.page_size : 128;
    CUtensorMap tq, tk, tv;
    if (!make_tmap_heads_bf16(&tq, a.q, HD, a.H, (uint64_t)a.B * a.n_q, a.q_ld, p.s.grp, p.tt1) ||
        !make_tmap_bf16(&tk, a.k, rows, cols, box) || !make_tmap_bf16(&tv, a.v, rows, cols, box))
        return cudaErrorInvalidValue;
    return launch_pdl(branch_attn_kernel<HD, QT>, dim3(p.s.G), dim3(A::THREADS), A::SMEM_BYTES, st, tq, tk, tv,
                      reinterpret_cast<bf16 *>(a.o), a.o_ld, sl2, p.tt1, p.s, err);
}
template <int HD>
static cudaError_t launch_f32(const BranchAttnArgs &a, const BranchPlan &p, float sl2, int *err, cudaStream_t st) {
    using A = BranchTileF32<HD>;
    static DeviceSet asked{0};
    cudaError_t e = allow_smem(branch_attn_f32_kernel<HD>, A::SMEM_BYTES, asked);
    if (e != cudaSuccess) return e;
    return launch_pdl(branch_attn_f32_kernel<HD>, dim3(p.s.G), dim3(256), A::SMEM_BYTES, st,
                      reinterpret_cast<const float *>(a.q), a.q_ld, reinterpret_cast<const float *>(a.k),
                      reinterpret_cast<const float *>(a.v), reinterpret_cast<float *>(a.o), a.o_ld, sl2, p.s, err);
}
template <typename T, int HD>
static cudaError_t launch_combine(const BranchAttnArgs &a, const BranchPlan &p, cudaStream_t st) {
    T *o = reinterpret_cast<T *>(a.o);
    if (p.s.n_pr > 0) {
        constexpr int RB = COMBINE_THREADS / (HD / 4), RS = COMBINE_SMALL / (HD / 4);
        const unsigned units = (unsigned)(p.s.Hk * p.s.E);
        const long prefixes = (long)p.s.Hk * p.s.n_pr;
        auto launch = [&](auto kernel, int threads, int rb) {
            return launch_pdl(kernel, dim3(units, (p.s.pitch_o + rb - 1) / rb), dim3(threads), 0, st, o, a.o_ld, p.s);
        };
        // 4 pieces at a time where a prefix row has 5 or fewer: 8 branches of 600
        // tokens over 16000 keys, 16 / 8 heads x 128 539 -> 521 us, 32 of 40 over 2048
        // 94 -> 85; but 32 single tokens over 38880 (19 pieces) 63.7 -> 64.9.
        const bool few = p.s.G <= 5 * prefixes;
        // CTAs of 64 threads where an entry's rows would leave half of 256 idle,
        // if the entries are more than one round of CTAs, or a row's pieces few
        // enough (8 a thread) for the few shares: 200 single tokens over 256 keys,
        // 32 / 8 heads x 128 69 -> 63 us, 16 / 8 heads x 64 58 -> 49; but 4 single
        // tokens over 32768 keys, one head x 128 16.8 -> 21.5.
        const int shares = p.s.pitch_o < RS ? RS / p.s.pitch_o : 1;
        if (2 * p.s.pitch_o <= RB && (units > 3u * device_sms() || p.s.G <= 8 * shares * prefixes))
            return few ? launch(branch_combine_kernel<T, HD, true, COMBINE_SMALL, 4>, COMBINE_SMALL, RS)
                       : launch(branch_combine_kernel<T, HD, true, COMBINE_SMALL, 8>, COMBINE_SMALL, RS);
        return few ? launch(branch_combine_kernel<T, HD, true, COMBINE_THREADS, 4>, COMBINE_THREADS, RB)
                   : launch(branch_combine_kernel<T, HD, true, COMBINE_THREADS, 8>, COMBINE_THREADS, RB);
    }
    constexpr int ROWS = 4 * COMBINE_THREADS / (HD / 4);
    if (p.s.G == 1) return cudaSuccess;
    return launch_pdl(branch_combine_kernel<T, HD, false, COMBINE_THREADS, 2>, dim3((unsigned)(p.s.G - 1), (p.s.pitch_o + ROWS - 1) / ROWS),
                      dim3(COMBINE_THREADS), 0, st, o, a.o_ld, p.s);
}

cudaError_t branch_attn(const xc_kv_cache &c, const BranchAttnArgs &a, void *ws, int *err, cudaStream_t st) {
    BranchPlan p = branch_plan(c, a.B, a.n_q, a.H, a.shared);
    p.s.seqs = a.seqs;
    p.s.causal = a.causal;
    p.s.shared = a.shared;
    p.s.lse = a.lse;
    p.s.ws_start = reinterpret_cast<int4 *>(ws);
    p.s.ws_o = reinterpret_cast<float *>(p.s.ws_start + p.s.G);
    p.s.ws_ml = reinterpret_cast<float2 *>(p.s.ws_o + p.rows * c.head_dim);
    p.s.ws_off = reinterpret_cast<int *>(p.s.ws_ml + p.rows);
    const float sl2 = a.scale * 1.4426950408889634f;
    cudaError_t e = cudaErrorInvalidValue;
    if (c.dtype == XC_BF16) {
        if (c.head_dim == 64) e = p.qt == 2 ? launch_tc<64, 2>(c, a, p, sl2, err, st) : launch_tc<64, 1>(c, a, p, sl2, err, st);
        if (c.head_dim == 128) e = p.qt == 2 ? launch_tc<128, 2>(c, a, p, sl2, err, st) : launch_tc<128, 1>(c, a, p, sl2, err, st);
        if (e != cudaSuccess) return e;
        return c.head_dim == 64 ? launch_combine<bf16, 64>(a, p, st) : launch_combine<bf16, 128>(a, p, st);
    }
    switch (c.head_dim) {
        case 16: e = launch_f32<16>(a, p, sl2, err, st); return e != cudaSuccess ? e : launch_combine<float, 16>(a, p, st);
        case 32: e = launch_f32<32>(a, p, sl2, err, st); return e != cudaSuccess ? e : launch_combine<float, 32>(a, p, st);
        case 64: e = launch_f32<64>(a, p, sl2, err, st); return e != cudaSuccess ? e : launch_combine<float, 64>(a, p, st);
        case 128: e = launch_f32<128>(a, p, sl2, err, st); return e != cudaSuccess ? e : launch_combine<float, 128>(a, p, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace xc
