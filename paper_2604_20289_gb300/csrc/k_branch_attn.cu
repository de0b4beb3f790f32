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

struct BranchSched {
    int B, n_q, grp, Hk;
    int tt;                  // tokens of a row tile
    int n_pr, n_pt;          // prefix row tiles and key tiles (n_pr = 0: no prefix units)
    int n_st, E;             // own row tiles per branch, of all branches
    int P;                   // keys of the prefix units: own keys begin there
    int causal, G;           // G: CTAs
    int max_seqs, max_pages, ps, n_pages;
    int pitch_p, pitch_o;    // rows of a partial slot
    long slots_p;            // prefix slots before the own ones
    const int *seqs, *len, *table;
    float *ws_o;             // partial O rows, then (m, l) of each, then the scan
    float2 *ws_ml;
    int *ws_off;             // [E + 1] own key tiles before each entry (same for every head)

    __host__ __device__ __forceinline__ int seq(int b) const {
        const int s = seqs[b];
        return s >= 0 && s < max_seqs ? s : -1;
    }
    __host__ __device__ __forceinline__ int seq_len(int b) const {
        const int s = seq(b);
        const int l = s < 0 ? 0 : len[s];
        return l < 0 || l > max_pages * ps ? 0 : l;
    }
    // keys that query i of a branch of length l sees
    __host__ __device__ __forceinline__ int limit(int l, int i) const {
        const int x = causal ? l - n_q + i + 1 : l;
        return x > 0 ? x : 0;
    }
    // keys past P that the entry's last row sees
    __host__ __device__ __forceinline__ int own_keys(int e) const {
        const int b = e / n_st, i = min((e - b * n_st + 1) * tt, n_q) - 1;
        return max(limit(seq_len(b), i) - P, 0);
    }
    // CTA c runs the key tiles [begin(c), begin(c + 1)); with fewer tiles than
    // CTAs the first T of them run one each
    __host__ __device__ __forceinline__ long long begin(long long T, int c) const {
        return T < G ? min((long long)c, T) : T * c / G;
    }
    __host__ __device__ __forceinline__ int owner(long long T, long long x) const {
        return T < G ? (int)x : (int)(((x + 1) * G - 1) / T);
    }
};

// One piece of a unit, as every role of a CTA walks them.
struct BranchPiece {
    int h, t0, nt;           // key head, first token row, tokens
    int row;                 // row of the page table, or -1
    int key0, keys;          // first key and keys of the unit
    int kt0, kt1, n_kt;      // key tiles of the piece and of the unit
    int idx;                 // unit of the head: prefix tiles, then entries
};
struct BranchStart {
    long long T;
    int h, idx, off, n;      // first unit, key tile in it, key tiles of this CTA
};

template <int KT>
struct BranchWalk {
    const BranchSched &s;
    int h, idx, off, left;
    __host__ __device__ __forceinline__ BranchWalk(const BranchSched &sc, const BranchStart &st)
        : s(sc), h(st.h), idx(st.idx), off(st.off), left(st.n) {}
    __host__ __device__ __forceinline__ bool next(BranchPiece &p) {
        while (left > 0) {
            int keys;
            if (idx < s.n_pr) {
                keys = s.P;
                p.n_kt = s.n_pt;
            } else {
                keys = s.own_keys(idx - s.n_pr);
                p.n_kt = (keys + KT - 1) / KT;
            }
            if (off < p.n_kt) {
                p.h = h;
                p.idx = idx;
                p.keys = keys;
                if (idx < s.n_pr) {
                    p.t0 = idx * s.tt;
                    p.nt = min(s.tt, s.B * s.n_q - p.t0);
                    p.row = s.seq(0);
                    p.key0 = 0;
                } else {
                    const int e = idx - s.n_pr, b = e / s.n_st, i0 = (e - b * s.n_st) * s.tt;
                    p.t0 = b * s.n_q + i0;
                    p.nt = min(s.tt, s.n_q - i0);
                    p.row = s.seq(b);
                    p.key0 = s.P;
                }
                p.kt0 = off;
                p.kt1 = min(p.n_kt, off + left);
                left -= p.kt1 - p.kt0;
                off = p.kt1;
                return true;
            }
            off = 0;
            if (++idx == s.n_pr + s.E) {
                idx = 0;
                ++h;
            }
        }
        return false;
    }
};

// This CTA's share of the line.  Every thread calls it; sh holds 34 ints.
// CTA 0 also leaves the entries' scan for the combine kernel.
template <int KT>
__device__ BranchStart branch_start(const BranchSched &s, int *sh, BranchStart *out, int *err) {
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = nt >> 5;
    const int per = (s.E + nt - 1) / nt;
    const int e0 = min(tid * per, s.E), e1 = min(e0 + per, s.E);
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += (s.own_keys(e) + KT - 1) / KT;
    int x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) sh[warp] = x;
    if (tid == 0) out->n = 0;
    __syncthreads();
    int before = 0, S = 0;
    for (int w = 0; w < nw; ++w) {
        if (w < warp) before += sh[w];
        S += sh[w];
    }
    const int excl = before + x - mine;
    const long long PP = (long long)s.n_pr * s.n_pt, Th = PP + S, T = Th * s.Hk;
    const int c = blockIdx.x;
    if (c == 0) {
        int a = excl;
        for (int e = e0; e < e1; ++e) {
            s.ws_off[e] = a;
            a += (s.own_keys(e) + KT - 1) / KT;
        }
        if (tid == 0) s.ws_off[s.E] = S;
        for (int b = tid; b < s.B; b += nt) {          // what the host could not see
            const int q = s.seqs[b];
            if (err && (q < 0 || q >= s.max_seqs || s.len[q] < 0 || s.len[q] > s.max_pages * s.ps || s.len[q] < s.P))
                atomicOr(err, ERR_BAD_SEQ);
        }
    }
    if (T > 0) {
        const long long g0 = s.begin(T, c), g1 = s.begin(T, c + 1);
        if (g1 > g0) {
            const int h = (int)(g0 / Th);
            const long long r = g0 - (long long)h * Th;
            if (r < PP) {
                if (tid == 0) *out = BranchStart{T, h, (int)(r / s.n_pt), (int)(r % s.n_pt), (int)(g1 - g0)};
            } else if (r - PP >= excl && r - PP < excl + mine) {
                int rest = (int)(r - PP) - excl, e = e0;
                for (;; ++e) {
                    const int n = (s.own_keys(e) + KT - 1) / KT;
                    if (rest < n) break;
                    rest -= n;
                }
                *out = BranchStart{T, h, s.n_pr + e, rest, (int)(g1 - g0)};
            }
        }
    }
    __syncthreads();
    return *out;
}

// Partial slot of a piece: with prefix units, unit index + CTA (both only
// grow along the line, so the sum names the piece); without, a CTA cuts at
// most its first and its last unit.
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
    static constexpr int STAGES = HD == 64 ? (QT == 2 ? 4 : 5) : (QT == 2 ? 2 : 3);
    static constexpr int OFF_K = QT * Q_BYTES, OFF_V = OFF_K + STAGES * KV_BYTES;
    static constexpr int OFF_BAR = OFF_V + STAGES * KV_BYTES;
    static constexpr int SMEM_BYTES = OFF_BAR + 640 + 1024;
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
__device__ __forceinline__ float exp2_mufu(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *tm, uint64_t *bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

// Warps: 4 QT softmax (thread = row of a 128-row tile = TMEM lane), one that
// loads (Q of a piece, then 128-key K and V tiles, page by page, by TMA), the
// MMA issuers (one per row tile where P has its own TMEM columns, else one),
// and one that clears the value rows past a unit's last key, whose weights are
// zero but whose bytes may be anything.
template <int HD, int QT>
__global__ void __launch_bounds__(BranchTile<HD, QT>::THREADS, 1)
    branch_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, bf16 *o, const long o_ld, const float sl2,
                       const int tt1, const __grid_constant__ BranchSched sc, int *err) {
    using A = BranchTile<HD, QT>;
    pdl_wait();
    extern __shared__ uint8_t smem_raw[];
    __shared__ int sh_scan[32];
    __shared__ BranchStart sh_start;
    const BranchStart start = branch_start<128>(sc, sh_scan, &sh_start, err);
    if (start.n == 0) return;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t *sQ = smem, *sK = smem + A::OFF_K, *sV = smem + A::OFF_V;
    uint64_t *bar = reinterpret_cast<uint64_t *>(smem + A::OFF_BAR);
    uint64_t *q_full = bar;                    // Q of piece p landed
    uint64_t *q_empty = bar + 1;               // every S of piece p done
    uint64_t *k_full = bar + 2;
    uint64_t *k_empty = k_full + A::STAGES;
    uint64_t *v_full = k_empty + A::STAGES;    // landed, and cleared past the last key
    uint64_t *v_empty = v_full + A::STAGES;
    uint64_t *v_tail = v_empty + A::STAGES;    // a unit's last V tile landed
    uint64_t *s_full = v_tail + A::STAGES;     // [QT] S_i computed
    uint64_t *s_cons = s_full + QT;            // [QT] S_i read (SEP_P)
    uint64_t *p_full = s_cons + QT;            // [QT] P_i written, O_i corrected
    uint64_t *pv_done = p_full + QT;           // [QT] P_i V done (SEP_P: every tile; else last of a piece)
    uint64_t *o_free = pv_done + QT;           // [QT] O_i of piece p read out
    uint64_t *turn = o_free + QT;              // [2][4] exponential-phase hand-off (TURNS)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(turn + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, A::ISSUERS);
        for (int s = 0; s < A::STAGES; ++s) {
            mbar_init(&k_full[s], 1);
            mbar_init(&k_empty[s], A::ISSUERS);
            mbar_init(&v_full[s], 1);
            mbar_init(&v_empty[s], A::ISSUERS);
            mbar_init(&v_tail[s], 1);
        }
        for (int i = 0; i < QT; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_cons[i], 128);
            mbar_init(&p_full[i], 128);
            mbar_init(&pv_done[i], 1);
            mbar_init(&o_free[i], 128);
        }
        for (int i = 0; i < 8; ++i) mbar_init(&turn[i], 1);
        mbar_fence_init();
    }
    if (warp == A::W_MMA) tmem_alloc(tmem_slot, A::TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    BranchWalk<128> walk(sc, start);
    BranchPiece pc;

    if (warp == A::W_TMA) {
        // ------------------------------------------------------ TMA producer
        const int box = min(sc.ps, 128), log_ps = 31 - __clz(sc.ps);
        const int q_bytes = QT * A::NR * tt1 * sc.grp * 128;
        int p = 0, g = 0;
        uint32_t tails = 0, tail_ph = 0;       // stages whose last use was a tail, parity of their tail uses
        bool ok = true;
        while (ok && walk.next(pc)) {
            if (p > 0) ok = mbar_wait(q_empty, (p - 1) & 1, err, ERR_WAIT_PRODUCER);
            if (!ok) break;
            if (lane == 0) {
                mbar_expect_tx(q_full, q_bytes);
                for (int i = 0; i < QT; ++i)
                    for (int r = 0; r < A::NR; ++r)
                        tma_load_3d(sQ + i * A::Q_BYTES + r * A::REGION, &tmQ, q_full, 64 * r, pc.h * sc.grp,
                                    pc.t0 + i * tt1);
            }
            ++p;
            const int *pages = sc.table + (size_t)max(pc.row, 0) * sc.max_pages;
            // first pool row of this lane's page in key tile kt (lane < pages of a tile)
            auto page_row = [&](int kt) {
                const int key = pc.key0 + kt * 128 + lane * box;
                if (lane * box >= 128 || kt * 128 + lane * box >= pc.keys || pc.row < 0) return -1;
                const int id = pages[key >> log_ps];
                if (id < 0 || id >= sc.n_pages) {
                    if (err) atomicOr(err, ERR_BAD_SEQ);
                    return sc.n_pages * sc.ps;         // out of range: TMA fills zeros
                }
                return id * sc.ps + (key & (sc.ps - 1));
            };
            int nrow = page_row(pc.kt0);
            for (int kt = pc.kt0; kt < pc.kt1; ++kt, ++g) {
                const int row = nrow;
                if (kt + 1 < pc.kt1) nrow = page_row(kt + 1);
                const int st = g % A::STAGES;
                const uint32_t ph = ((g / A::STAGES) & 1) ^ 1;
                const int n_pg = __popc(__ballot_sync(0xffffffffu, row >= 0));
                const uint32_t bytes = n_pg * box * 128 * A::NR;
                const bool tail = pc.keys < (kt + 1) * 128;
                ok = mbar_wait(&k_empty[st], ph, err, ERR_WAIT_PRODUCER);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                if (lane == 0) mbar_expect_tx(&k_full[st], bytes);
                __syncwarp();
                if (row >= 0)
                    for (int r = 0; r < A::NR; ++r)
                        tma_load_2d(sK + st * A::KV_BYTES + r * A::REGION + lane * box * 128, &tmK, &k_full[st],
                                    pc.h * HD + 64 * r, row);
                ok = mbar_wait(&v_empty[st], ph, err, ERR_WAIT_PRODUCER);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                uint64_t *vb = tail ? &v_tail[st] : &v_full[st];
                if (lane == 0) mbar_expect_tx(vb, bytes);
                __syncwarp();
                if (row >= 0)
                    for (int r = 0; r < A::NR; ++r)
                        tma_load_2d(sV + st * A::KV_BYTES + r * A::REGION + lane * box * 128, &tmV, vb,
                                    pc.h * HD + 64 * r, row);
                if (tail) tail_ph ^= 1u << st;
                tails = tail ? tails | 1u << st : tails & ~(1u << st);
            }
        }
        // every copy this warp started has landed before the CTA exits
        if (lane == 0) {
            if (p > 0) mbar_wait(q_full, (p - 1) & 1, err, ERR_WAIT_PRODUCER);
            for (int x = max(g - A::STAGES, 0); x < g; ++x) {
                const int st = x % A::STAGES;
                mbar_wait(&k_full[st], (x / A::STAGES) & 1, err, ERR_WAIT_PRODUCER);
                if (tails >> st & 1u) mbar_wait(&v_tail[st], (tail_ph >> st & 1u) ^ 1u, err, ERR_WAIT_PRODUCER);
                else mbar_wait(&v_full[st], (x / A::STAGES) & 1, err, ERR_WAIT_PRODUCER);
            }
        }
    } else if (warp == A::W_TAIL) {
        // -------------------------------- clears V rows past the last key
        uint32_t ph = 0;
        int g = 0;
        bool ok = true;
        while (ok && walk.next(pc)) {
            const int kt = pc.kt1 - 1;
            g += pc.kt1 - pc.kt0;
            const int valid = pc.keys - kt * 128;
            if (valid >= 128) continue;
            const int st = (g - 1) % A::STAGES;
            ok = mbar_wait(&v_tail[st], ph >> st & 1u, err, ERR_WAIT_PRODUCER);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ph ^= 1u << st;
            // rows are 128 bytes in each region whatever the swizzle of their 16-byte pieces
            for (int r = 0; r < A::NR; ++r)
                for (int x = max(valid, 0) * 8 + lane; x < 128 * 8; x += 32)
                    *reinterpret_cast<uint4 *>(sV + st * A::KV_BYTES + r * A::REGION + x * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_full[st]);
        }
    } else if (warp >= A::W_MMA) {
        // ------------------------------------------------------ MMA issue
        // The warp runs converged; one elected lane issues each instruction.
        constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false);
        constexpr uint32_t idesc_o = idesc_bf16(128, HD, false, true);
        const uint64_t dQ0 = sdesc_sw128(smem_u32(sQ), 16, 1024);
        const uint64_t dK0 = sdesc_sw128(smem_u32(sK), 16, 1024);
        const uint64_t dV0 = sdesc_sw128(smem_u32(sV), A::REGION, 1024);
        auto issue_s = [&](int i, int g) {             // S_i = Q_i K_g^T
            const uint64_t dq = dQ0 + (uint64_t)((i * A::Q_BYTES) >> 4);
            const uint64_t dk = dK0 + (uint64_t)(((g % A::STAGES) * A::KV_BYTES) >> 4);
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
                const uint32_t off = ((ks >> 2) * A::REGION + (ks & 3) * 32) >> 4;
                tc_mma_warp(tmem + A::S_COL(i), dq + off, dk + off, idesc_s, ks > 0 ? 1u : 0u);
            }
            tc_commit_warp(&s_full[i]);
        };
        auto issue_pv = [&](int i, int g, bool fresh) {   // O_i (+)= P_i V_g, P_i in TMEM
            const uint64_t dv = dV0 + (uint64_t)(((g % A::STAGES) * A::KV_BYTES) >> 4);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                tc_mma_tmem_a_warp(tmem + A::O_COL(i), tmem + A::P_COL(i) + 8 * ks, dv + ((ks * 16 * 128) >> 4), idesc_o,
                                   (!fresh || ks > 0) ? 1u : 0u);
        };
        auto wait = [&](uint64_t *b, int parity) -> bool {
            const bool r = mbar_wait(b, parity & 1, err, ERR_WAIT_MMA);
            return __all_sync(0xffffffffu, r) != 0;
        };
        // The key tiles of the CTA as two walks, S one tile ahead of P V.
        struct Tile {
            int g, p;                                  // tile and piece of the CTA
            bool first, last;                          // of its piece
        };
        BranchWalk<128> walk_s = walk;
        BranchPiece ps{}, pv{};
        Tile ts{-1, -1, false, true}, tv{-1, -1, false, true};
        auto step = [&](BranchWalk<128> &w, BranchPiece &c, Tile &t) -> bool {
            if (t.last) {
                if (!w.next(c)) return false;
                ++t.p;
                t.first = true;
            } else {
                ++c.kt0;
                t.first = false;
            }
            ++t.g;
            t.last = c.kt0 == c.kt1 - 1;
            return true;
        };
        auto s_ready = [&](const Tile &t) -> bool {
            if (t.first && !wait(q_full, t.p)) return false;
            return wait(&k_full[t.g % A::STAGES], t.g / A::STAGES);
        };
        auto pv_ready = [&](int i, const Tile &t) -> bool {
            if (t.first && t.p > 0 && !wait(&o_free[i], t.p - 1)) return false;
            return wait(&p_full[i], t.g) && wait(&v_full[t.g % A::STAGES], t.g / A::STAGES);
        };
        if constexpr (A::SEP_P) {
            // S_i of the next tile as soon as the softmax has read S_i, then
            // P_i V once P_i is ready
            const int i = warp - A::W_MMA;
            bool more = step(walk_s, ps, ts);
            bool ok = s_ready(ts);
            if (ok) {
                tc_fence_after();
                issue_s(i, 0);
                tc_commit_warp(&k_empty[0]);
                if (ts.last) tc_commit_warp(q_empty);
            }
            while (ok && step(walk, pv, tv)) {
                more = more && step(walk_s, ps, ts);
                if (more) {
                    if (!(wait(&s_cons[i], tv.g) && s_ready(ts))) break;
                    tc_fence_after();
                    issue_s(i, ts.g);
                    tc_commit_warp(&k_empty[ts.g % A::STAGES]);
                    if (ts.last) tc_commit_warp(q_empty);
                }
                if (!pv_ready(i, tv)) break;
                tc_fence_after();
                issue_pv(i, tv.g, tv.first);
                tc_commit_warp(&pv_done[i]);
                tc_commit_warp(&v_empty[tv.g % A::STAGES]);
            }
        } else {
            // P_i overwrites S_i: P0 V, next S0, P1 V, next S1 -- the order in
            // which the warpgroups finish
            bool more = step(walk_s, ps, ts);
            bool ok = s_ready(ts);
            if (ok) {
                tc_fence_after();
                issue_s(0, 0);
                issue_s(1, 0);
                tc_commit_warp(&k_empty[0]);
                if (ts.last) tc_commit_warp(q_empty);
            }
            while (ok && step(walk, pv, tv)) {
                more = more && step(walk_s, ps, ts);
                if (!pv_ready(0, tv)) break;
                tc_fence_after();
                issue_pv(0, tv.g, tv.first);
                if (tv.last) tc_commit_warp(&pv_done[0]);
                if (more) {
                    if (!s_ready(ts)) break;
                    tc_fence_after();
                    issue_s(0, ts.g);
                }
                if (!pv_ready(1, tv)) break;
                tc_fence_after();
                issue_pv(1, tv.g, tv.first);
                tc_commit_warp(&v_empty[tv.g % A::STAGES]);
                if (tv.last) tc_commit_warp(&pv_done[1]);
                if (more) {
                    issue_s(1, ts.g);
                    tc_commit_warp(&k_empty[ts.g % A::STAGES]);
                    if (ts.last) tc_commit_warp(q_empty);
                }
            }
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
        // running sum l.  cols: keys of this tile the row sees.  false: a wait
        // ran out.
        auto tile = [&](int g, int cols, bool fresh, bool live, float &m, float &l) -> bool {
            bool ok = mbar_wait(&s_full[wg], g & 1, err, ERR_WAIT_SOFTMAX);
            if (!__all_sync(0xffffffffu, ok)) return false;
            tc_fence_after();
            float s[128];
            float alpha = 1.0f;
            bool grow = false;
            if (live) {
                tmem_ld128_sync(tS, s);
                if constexpr (A::SEP_P) {
                    tc_fence_before();
                    mbar_arrive(&s_cons[wg]);
                }
                if (__any_sync(0xffffffffu, cols < 128)) {
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
                // a row that sees no key of a piece's first tile sees none of
                // the piece: m stays -inf, every weight 0
                if (fresh) m = m_new;
                grow = !fresh && m_new > m + A::LAZY;
                if (grow) {
                    alpha = exp2_mufu(m - m_new);
                    m = m_new;
                }
            } else if constexpr (A::SEP_P) {
                mbar_arrive(&s_cons[wg]);
            }
            if constexpr (A::SEP_P) {
                // P_i free and O_i stable once P V of the previous tile is done
                if (g >= 1) {
                    ok = mbar_wait(&pv_done[wg], (g - 1) & 1, err, ERR_WAIT_SOFTMAX);
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
                    if (!__all_sync(0xffffffffu, ok)) return false;
                }
            }
            if (live) {
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
                }
                const float2 rs = __fadd2_rn(rs0, rs1);
                l = l * alpha + (rs.x + rs.y);
            }
            tc_fence_before();
            mbar_arrive(&p_full[wg]);
            if constexpr (A::TURNS) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&turn[4 * (wg ^ 1) + q]);
            }
            return true;
        };
        int g = 0, p = 0;
        bool ok = true;
        while (ok && walk.next(pc)) {
            const bool row_ok = in_tile && tl_ < pc.nt;
            const bool live = __any_sync(0xffffffffu, row_ok) != 0;
            const int t = pc.t0 + tl_;
            int see = 1 << 30;                             // keys of the unit this row sees
            if (row_ok) {
                const int b = t / sc.n_q;
                see = min(sc.limit(sc.seq_len(b), t - b * sc.n_q) - pc.key0, pc.keys);
            }
            float m = -INFINITY, l = 0.0f;
            for (int kt = pc.kt0; kt < pc.kt1; ++kt, ++g) {
                ok = tile(g, see - kt * 128, kt == pc.kt0, live, m, l);
                if (!ok) break;
            }
            if (!ok) break;
            ok = mbar_wait(&pv_done[wg], (A::SEP_P ? g - 1 : p) & 1, err, ERR_WAIT_SOFTMAX);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (live) {
                if (sc.n_pr == 0 && pc.kt1 - pc.kt0 == pc.n_kt) {
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    bf16 *dst = o + (size_t)t * o_ld + (pc.h * sc.grp + gq) * HD;
#pragma unroll 1
                    for (int c = 0; c < HD / 16; ++c) {
                        float x[16];
                        tmem_ld16_sync(tO + 16 * c, x);
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] *= inv;
                        if (row_ok) store16<bf16>(dst + 16 * c, x);
                    }
                } else {
                    const long row = branch_slot_row(sc, pc, blockIdx.x, p == 0) + tl_ * sc.grp + gq;
#pragma unroll 1
                    for (int c = 0; c < HD / 16; ++c) {
                        float x[16];
                        tmem_ld16_sync(tO + 16 * c, x);
                        if (row_ok) store16<float>(sc.ws_o + row * HD + 16 * c, x);
                    }
                    if (row_ok) sc.ws_ml[row] = make_float2(m, l);
                }
            }
            tc_fence_before();
            mbar_arrive(&o_free[wg]);
            ++p;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == A::W_MMA) {
        tc_fence_after();
        tmem_dealloc(tmem, A::TMEM_COLS);
    }
}

// ------------------------------------------------------------ fp32 kernel
// 64-row x 64-key tiles, 256 threads as 16 x 16: thread (ty, tx) computes
// scores of rows 4 ty.. and keys tx + 16 j, and the same rows' output columns
// tx + 16 j.  fp32 FMA bound; exact exp2f, no bf16 anywhere.
template <int HD>
struct BranchTileF32 {
    static constexpr int RT = 64, KT = 64, LD = HD + 4, LDP = KT + 4;
    static constexpr int SMEM_BYTES = (3 * 64 * LD + 64 * LDP) * (int)sizeof(float);
};
template <int HD>
__global__ void __launch_bounds__(256)
    branch_attn_f32_kernel(const float *q, const long q_ld, const float *__restrict__ k, const float *__restrict__ v,
                           float *o, const long o_ld, const float sl2, const __grid_constant__ BranchSched sc, int *err) {
    using A = BranchTileF32<HD>;
    pdl_wait();
    extern __shared__ __align__(16) float sm[];
    __shared__ int sh_scan[32];
    __shared__ BranchStart sh_start;
    const BranchStart start = branch_start<64>(sc, sh_scan, &sh_start, err);
    float *sQ = sm, *sK = sQ + 64 * A::LD, *sV = sK + 64 * A::LD, *sP = sV + 64 * A::LD;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int log_ps = 31 - __clz(sc.ps);
    const size_t ld = (size_t)sc.Hk * HD;
    constexpr int V4 = HD / 4;                             // float4 of a row
    constexpr int NC = HD / 16;                            // output columns of a thread
    BranchWalk<64> walk(sc, start);
    BranchPiece pc;
    int np = 0;
    while (walk.next(pc)) {
        const int rows = pc.nt * sc.grp;
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
        float m[4], l[4], acc[4][NC];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i;
            see[i] = 0;
            if (r < rows) {
                const int t = pc.t0 + r / sc.grp, b = t / sc.n_q;
                see[i] = min(sc.limit(sc.seq_len(b), t - b * sc.n_q) - pc.key0, pc.keys);
            }
            m[i] = -INFINITY;
            l[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < NC; ++j) acc[i][j] = 0.0f;
        }
        for (int kt = pc.kt0; kt < pc.kt1; ++kt) {
            __syncthreads();
            for (int x = tid; x < 64 * V4; x += 256) {
                const int r = x / V4, c = x % V4, key = kt * 64 + r;
                float4 fk = make_float4(0, 0, 0, 0), fv = fk;
                if (key < pc.keys && pc.row >= 0) {
                    const int at = pc.key0 + key;
                    const int id = sc.table[(size_t)pc.row * sc.max_pages + (at >> log_ps)];
                    if (id >= 0 && id < sc.n_pages) {
                        const size_t off = ((size_t)id * sc.ps + (at & (sc.ps - 1))) * ld + pc.h * HD + 4 * c;
                        fk = *reinterpret_cast<const float4 *>(k + off);
                        fv = *reinterpret_cast<const float4 *>(v + off);
                    } else if (err) {
                        atomicOr(err, ERR_BAD_SEQ);
                    }
                }
                *reinterpret_cast<float4 *>(sK + r * A::LD + 4 * c) = fk;
                *reinterpret_cast<float4 *>(sV + r * A::LD + 4 * c) = fv;
            }
            __syncthreads();
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
#pragma unroll
                    for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    l[i] = l[i] * alpha + sum;
                    m[i] = mn;
#pragma unroll
                    for (int j = 0; j < NC; ++j) acc[i][j] *= alpha;
                }
                __syncwarp();                              // a warp reads only its own rows of P
#pragma unroll 2
                for (int c = 0; c < 64; c += 4) {
                    float4 a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4 *>(sP + (4 * ty + i) * A::LDP + c);
#pragma unroll
                    for (int j = 0; j < NC; ++j) {
                        const float *b = sV + c * A::LD + tx + 16 * j;
                        const float b0 = b[0], b1 = b[A::LD], b2 = b[2 * A::LD], b3 = b[3 * A::LD];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[i][j] = fmaf(a[i].x, b0, acc[i][j]);
                            acc[i][j] = fmaf(a[i].y, b1, acc[i][j]);
                            acc[i][j] = fmaf(a[i].z, b2, acc[i][j]);
                            acc[i][j] = fmaf(a[i].w, b3, acc[i][j]);
                        }
                    }
                }
            }
        }
        const bool whole = sc.n_pr == 0 && pc.kt1 - pc.kt0 == pc.n_kt;
        const long row0 = whole ? 0 : branch_slot_row(sc, pc, blockIdx.x, np == 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i;
            if (r >= rows) continue;
            if (whole) {
                const float inv = l[i] > 0.0f ? 1.0f / l[i] : 0.0f;
                float *dst = o + (size_t)(pc.t0 + r / sc.grp) * o_ld + (pc.h * sc.grp + r % sc.grp) * HD;
#pragma unroll
                for (int j = 0; j < NC; ++j) dst[tx + 16 * j] = acc[i][j] * inv;
            } else {
#pragma unroll
                for (int j = 0; j < NC; ++j) sc.ws_o[(row0 + r) * HD + tx + 16 * j] = acc[i][j];
                if (tx == 0) sc.ws_ml[row0 + r] = make_float2(m[i], l[i]);
            }
        }
        ++np;
    }
}

// ---------------------------------------------------------------- combine
// grid.x = (key head, own entry), grid.y = 8 rows of it, one warp each.  Adds
// the pieces of the row's prefix unit and of its own unit in CTA order; rows
// already written are left, rows without keys get zeros.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
    branch_combine_kernel(T *o, const long o_ld, const __grid_constant__ BranchSched s) {
    pdl_wait();
    constexpr int W = HD >= 32 ? HD / 32 : 1;              // columns of a lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.x / s.E, e = blockIdx.x - h * s.E;
    const int b = e / s.n_st, i0 = (e - b * s.n_st) * s.tt;
    const int r = blockIdx.y * 8 + warp;
    if (r >= min(s.tt, s.n_q - i0) * s.grp) return;
    const long long Th = (long long)s.n_pr * s.n_pt + s.ws_off[s.E], Tl = Th * s.Hk;
    const int n_own = s.ws_off[e + 1] - s.ws_off[e];
    const int t = b * s.n_q + i0 + r / s.grp;
    int np = 0, no = 0, cp = 0, co = 0;                    // pieces and first CTA of both units
    long long so = 0;
    long row_p = 0;
    if (s.n_pr > 0) {
        const int pi = t / s.tt;
        const long long s0 = h * Th + (long long)pi * s.n_pt;
        cp = s.owner(Tl, s0);
        np = s.owner(Tl, s0 + s.n_pt - 1) - cp + 1;
        row_p = ((long)h * s.n_pr + pi) * s.pitch_p + (t - pi * s.tt) * s.grp + r % s.grp;
    }
    if (n_own > 0) {
        so = h * Th + (long long)s.n_pr * s.n_pt + s.ws_off[e];
        co = s.owner(Tl, so);
        no = s.owner(Tl, so + n_own - 1) - co + 1;
        if (s.n_pr == 0 && no == 1) return;                // written by the CTA that ran it whole
    }
    auto row_of = [&](int k) -> long {                     // partial row of the k-th piece
        if (k < np) return row_p + (long)(cp + k) * s.pitch_p;
        const int c = co + k - np;
        if (s.n_pr > 0) return s.slots_p * s.pitch_p + ((long)h * s.E + e + c) * s.pitch_o + r;
        return (2l * c + (s.begin(Tl, c) >= so ? 0 : 1)) * s.pitch_o + r;
    };
    const int n = np + no;
    float mm = -INFINITY;
    for (int k = lane; k < n; k += 32) mm = fmaxf(mm, s.ws_ml[row_of(k)].x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
    float den = 0.0f, acc[W];
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = 0.0f;
    for (int k0 = 0; k0 < n; k0 += 32) {
        float w = 0.0f;
        long row = 0;
        if (k0 + lane < n) {
            row = row_of(k0 + lane);
            const float2 ml = s.ws_ml[row];
            w = ml.x == -INFINITY ? 0.0f : exp2f(ml.x - mm);
            den += w * ml.y;
        }
        const int m = min(32, n - k0);
#pragma unroll 4
        for (int k = 0; k < m; ++k) {
            const float wk = __shfl_sync(0xffffffffu, w, k);
            const long rk = __shfl_sync(0xffffffffu, row, k);
            if (wk == 0.0f || lane * W >= HD) continue;    // a piece without keys for this row
            const float *src = s.ws_o + rk * HD + lane * W;
            float x[W];
            if constexpr (W == 4) {
                const float4 f = *reinterpret_cast<const float4 *>(src);
                x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
            } else if constexpr (W == 2) {
                const float2 f = *reinterpret_cast<const float2 *>(src);
                x[0] = f.x; x[1] = f.y;
            } else {
                x[0] = src[0];
            }
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] = fmaf(wk, x[j], acc[j]);
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) den += __shfl_xor_sync(0xffffffffu, den, d);
    const float inv = den > 0.0f ? 1.0f / den : 0.0f;
    T *dst = o + (size_t)t * o_ld + (h * s.grp + r % s.grp) * HD + lane * W;
    if (lane * W < HD) {
#pragma unroll
        for (int j = 0; j < W; ++j) dst[j] = from_f<T>(acc[j] * inv);
    }
}

// ------------------------------------------------------------------- host
struct BranchPlan {
    BranchSched s;
    int qt, tt1, chunks;
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
    // two row tiles per CTA where a unit's rows can fill them
    const long long tokens = (long long)B * n_q;
    p.qt = !f32 && (shared > 0 ? tokens : (long long)n_q) > p.tt1 ? 2 : 1;
    s.tt = p.tt1 * p.qt;
    s.n_st = (n_q + s.tt - 1) / s.tt;
    s.E = B * s.n_st;
    // prefix units where packing the branches' rows saves a tenth of the row tiles
    const long long packed = (tokens + s.tt - 1) / s.tt;
    if (shared > 0 && packed * 10 <= (long long)s.E * 9) {
        s.P = shared;
        s.n_pr = (int)packed;
        s.n_pt = (shared + KT - 1) / KT;
    }
    s.pitch_p = (int)(tokens < s.tt ? tokens : s.tt) * s.grp;
    s.pitch_o = (n_q < s.tt ? n_q : s.tt) * s.grp;
    s.slots_p = s.n_pr > 0 ? (long)s.Hk * s.n_pr + s.G : 0;
    const size_t slots_o = s.n_pr > 0 ? (size_t)s.Hk * s.E + s.G : 2 * (size_t)s.G;
    p.rows = (size_t)s.slots_p * s.pitch_p + slots_o * s.pitch_o;
    p.chunks = (s.pitch_o + 7) / 8;
    p.bytes = p.rows * (c.head_dim * sizeof(float) + sizeof(float2)) + ((size_t)s.E + 1) * sizeof(int);
    return p;
}
bool branch_attn_fits(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    const BranchPlan p = branch_plan(c, B, n_q, H, shared);
    const long long kt = c.dtype == XC_F32 ? 64 : 128;
    const long long own = (long long)p.s.E * (((long long)c.max_pages * c.page_size + kt - 1) / kt);
    return (long long)B * ((n_q + p.s.tt - 1) / p.s.tt) < (1ll << 30) && p.s.Hk * ((long long)p.s.n_pr * p.s.n_pt + own) < (1ll << 31);
}
size_t branch_attn_workspace_bytes(const xc_kv_cache &c, int B, int n_q, int H, int shared) {
    return branch_plan(c, B, n_q, H, shared).bytes;
}

template <typename K> static cudaError_t allow_smem(K kernel, int bytes, bool &done) {
    if (done) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    done = e == cudaSuccess;
    return e;
}

template <int HD, int QT>
static cudaError_t launch_tc(const xc_kv_cache &c, const BranchAttnArgs &a, const BranchPlan &p, float sl2, int *err,
                             cudaStream_t st) {
    using A = BranchTile<HD, QT>;
    static bool done = false;
    cudaError_t e = allow_smem(branch_attn_kernel<HD, QT>, A::SMEM_BYTES, done);
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
    static bool done = false;
    cudaError_t e = allow_smem(branch_attn_f32_kernel<HD>, A::SMEM_BYTES, done);
    if (e != cudaSuccess) return e;
    return launch_pdl(branch_attn_f32_kernel<HD>, dim3(p.s.G), dim3(256), A::SMEM_BYTES, st,
                      reinterpret_cast<const float *>(a.q), a.q_ld, reinterpret_cast<const float *>(a.k),
                      reinterpret_cast<const float *>(a.v), reinterpret_cast<float *>(a.o), a.o_ld, sl2, p.s, err);
}
template <typename T, int HD>
static cudaError_t launch_combine(const BranchAttnArgs &a, const BranchPlan &p, cudaStream_t st) {
    return launch_pdl(branch_combine_kernel<T, HD>, dim3((unsigned)(p.s.Hk * p.s.E), p.chunks), dim3(256), 0, st,
                      reinterpret_cast<T *>(a.o), a.o_ld, p.s);
}

cudaError_t branch_attn(const xc_kv_cache &c, const BranchAttnArgs &a, void *ws, int *err, cudaStream_t st) {
    BranchPlan p = branch_plan(c, a.B, a.n_q, a.H, a.shared);
    p.s.seqs = a.seqs;
    p.s.causal = a.causal;
    p.s.ws_o = reinterpret_cast<float *>(ws);
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
