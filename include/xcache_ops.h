/*
 * xcache_ops.h -- operator-level entry points of the X-Cache hot path.
 *
 * These run ONE kernel of the chunk step on caller-owned device buffers, so
 * that each step of the path can be checked against the CPU oracle at full
 * size.  xc_chunk_step runs exactly these kernels.  All pointers are DEVICE
 * pointers; `stream` is a cudaStream_t (NULL = legacy default stream);
 * every call is asynchronous.  Activations use `dtype` (XC_F32: float32,
 * XC_BF16: bfloat16); vectors such as bias / gate / shift / scale are float32.
 * Weights are K-major: Wt [N][K] holds W^T of y = x W.
 * Errors: XC_EINVAL for a bad shape or pointer, XC_ECUDA for a launch
 * failure.  Kernels with bounded waits record expiry in a device error word
 * that xc_op_device_error() returns.
 */
#ifndef XCACHE_OPS_H
#define XCACHE_OPS_H

#include "xcache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    XC_EPI_BIAS = 0,        /* out = A W + b                                     */
    XC_EPI_GELU = 1,        /* out = GELU_tanh(A W + b)  (FFN up-projection)     */
    XC_EPI_RESID_GATE = 2,  /* out = resid + gate * (A W + b)  (adaLN-Zero gated
                               residual of Eq. 1; O-projection / FFN down)       */
    XC_EPI_RESID_CACHE = 3  /* as XC_EPI_RESID_GATE and additionally
                               rhat = round(out) - xin (block residual, Eq. 2-3) */
} xc_epilogue;

/* C[M][N] = epilogue(A[M][K] @ Wt[N][K]^T).  M >= 1; N % 256 == 0 and K % 64 == 0
 * for XC_BF16 (tcgen05 path), N % 16 == 0 for XC_F32.  `gate`, `resid`,
 * `xin`, `rhat` may be NULL when the epilogue does not use them. */
xc_status xc_op_linear(int dtype, int epilogue, int M, int N, int K, const void *A,
                       const void *Wt, const float *bias, const float *gate,
                       const void *resid, const void *xin, void *out, void *rhat,
                       void *stream);

/* QKV projection with RoPE (Section 2.1 block, reading of RoPE over
 * (camera, absolute frame, h, w)).  A [M][d] with M = n_cams*frames*gh*gw,
 * Wt [3d][d], bias [3d]; writes q, k, v [M][d] (heads interleaved by column:
 * head h owns columns h*head_dim ...).  Token row r of chunk `chunk` sits at
 * camera r / (frames*gh*gw), absolute frame chunk*frames + f, grid (h, w). */
xc_status xc_op_qkv_rope(int dtype, int n_cams, int frames, int gh, int gw, int chunk,
                         int d, int head_dim, float rope_theta, const void *A,
                         const void *Wt, const float *bias, void *q, void *k, void *v,
                         void *stream);

/* o = softmax(q k^T / sqrt(head_dim)) v per head, no mask (every query sees
 * every key: full attention within the chunk and over all resident cached
 * keys).  q, o [Lq][H*hd]; k, v [n_keys][H*hd] (bf16: 16-byte aligned rows).
 *   workspace  device, optional.  With at least
 *              xc_op_attention_workspace_bytes() bytes and more (head,
 *              256-query) units than SMs, the work is spread evenly over the
 *              SMs: either the (unit, key tile) space is cut into equal
 *              shares, or -- with 8 or more waves of units and the K / V of
 *              all heads larger than L2 -- whole units run in waves and only
 *              the remaining units are cut; a second kernel merges the
 *              partials of the cut units.  With NULL (or too small) every
 *              unit runs whole on one SM.  Contents on entry are ignored; it
 *              must not be shared by calls that overlap in time.
 * bf16 needs head_dim 64 or 128; fp32 head_dim 16, 32 or 64. */
size_t xc_op_attention_workspace_bytes(int dtype, int head_dim);
xc_status xc_op_attention(int dtype, int Lq, int n_keys, int n_heads, int head_dim,
                          const void *q, const void *k, const void *v, void *o,
                          void *workspace, size_t workspace_bytes, void *stream);

/* out = LayerNorm(x) * (1 + scale) + shift over rows of length d (no affine,
 * population variance, eps), adaLN-Zero modulation.  x, out [M][d]. */
xc_status xc_op_ln_mod(int dtype, int M, int d, float eps, const void *x,
                       const float *shift, const float *scale, void *out, void *stream);

/* Reuse path of Eq. 4: out = round(x + rhat), n elements. */
xc_status xc_op_residual_reuse(int dtype, long n, const void *x, const void *rhat, void *out,
                               void *stream);

/* Per-(t, b) gate state kept on the device (32 bytes): EMA of the cosine
 * (Eq. 8), has-history bit, consecutive-skip counter (Section 2.5 (4)),
 * cache-valid bit, and which half of the double-buffered cached fingerprint
 * is active. */
typedef struct {
    double ema;
    int has_hist, stale, valid, active;
    int pad[2];
} xc_gate_cell;

/* Bytes of device workspace xc_op_gate needs for this geometry on the current
 * device (the gate's grid splits each camera's rows over the device's SMs). */
size_t xc_op_gate_workspace_bytes(int dtype, int n_cams, int tokens_per_cam, int d);

/* One gate evaluation of one (t, b) cell (Section 2.3-2.5): fingerprint of the
 * block input x (spatial sample, per-camera token mean, action), min-cosine
 * s_cos (Eq. 5) and max token deviation d_max (Eq. 6) against the cached
 * fingerprint, adaptive threshold (Eq. 9), decision (Eq. 7), EMA (Eq. 8) and
 * staleness updates.
 *   x        device [n_cams * tokens_per_cam][d] activation dtype
 *   fp_rows  device int [n_cams][kfp]: token rows of the spatial sample
 *   phi      device float [2][n_cams*kfp*d + n_cams*d]: the two halves of the
 *            cached fingerprint (spatial entries, then per-camera means); the
 *            current fingerprint is written into the inactive half
 *   phi_act  device float [2][8]: cached action halves
 *   cell     device xc_gate_cell, updated in place
 *   action   host float [action_dim] (action_dim <= 8)
 *   mode     1 evaluate the gate, 0 refresh only (forced compute)
 *   step     denoising step t (strict step-0 threshold)
 *   gate     knobs (NULL = Table 1); replay_skip[0], when set, replaces the
 *            decision (decision-replay mode)
 *   flag     device uint8 decision (xc_decision); s_cos, d_max, tau device float
 *   workspace device, >= xc_op_gate_workspace_bytes(); its counters are
 *            cleared by the call (cudaMemsetAsync), nothing is allocated
 * Asynchronous on `stream`.  Errors: XC_EINVAL. */
xc_status xc_op_gate(int dtype, int n_cams, int tokens_per_cam, int d, const void *x, const int *fp_rows,
                     int kfp, float *phi, float *phi_act, xc_gate_cell *cell, const float *action,
                     int action_dim, int mode, int step, const xc_gate_params *gate, uint8_t *flag,
                     float *s_cos, float *d_max, float *tau, void *workspace, size_t workspace_bytes,
                     void *stream);

/* Allocation-free variant of xc_op_gate.  The paper has no counterpart; this
 * is an interface of this library, for callers that cannot call cudaMalloc
 * when they call in: a runtime that owns the only device allocator of the
 * process (a plugin or embedding host), code held to a device-memory budget
 * fixed at start-up, or a latency-critical loop where an allocation and the
 * device synchronisation it may bring are not acceptable.
 * Same arguments, checks and results as xc_op_gate minus the workspace: the
 * gate's scratch (per-CTA partial metrics and column sums, and the tickets)
 * lives in one file-scope device array of 1 MiB (GATE_STATIC_SCRATCH_BYTES)
 * that every GPU which loads the library keeps until the process exits.
 * Nothing is allocated or freed; the tickets are cleared with
 * cudaMemsetAsync on each call.
 * The first call on a device looks up the array's device address
 * (cudaGetSymbolAddress) and caches it for that device for the rest of the
 * process; that first call should come before any stream capture.  The
 * cached address belongs to the device's primary context: do not use this
 * entry point after cudaDeviceReset() on that device, or from a context other
 * than the primary one.
 * All calls share the one array and it keeps the last call's contents:
 * calls that overlap on the GPU (different streams, no ordering) race; calls
 * ordered on one stream are safe.
 * Errors: XC_EINVAL for bad arguments (as xc_op_gate) or a geometry whose
 * scratch exceeds 1 MiB (the message states the bytes needed), XC_ECUDA if
 * the device or the array's address cannot be obtained. */
xc_status xc_op_gate_static(int dtype, int n_cams, int tokens_per_cam, int d, const void *x,
                            const int *fp_rows, int kfp, float *phi, float *phi_act, xc_gate_cell *cell,
                            const float *action, int action_dim, int mode, int step,
                            const xc_gate_params *gate, uint8_t *flag, float *s_cos, float *d_max,
                            float *tau, void *stream);

/* ---- branched rollouts over a paged key / value cache ----
 *
 * Several sequences (the branches of a rollout: candidate actions from one
 * history) live in one pool of pages.  A page holds page_size consecutive
 * tokens' keys and values of every head; a sequence is a row of page ids and
 * a token count; sequences forked from one another share pages.  All of the
 * state is on the device and every call is asynchronous, so a whole planning
 * step (fork, extend, append, attend, free) needs no host synchronisation.
 *
 *   k, v   [n_layers][n_pages][page_size][n_kv_heads * head_dim], 16-byte aligned
 *   ref    [n_pages] sequences that hold the page; 0 = free
 *   table  [max_seqs][max_pages] page ids, token j of sequence s on page
 *          table[s][j / page_size]; entries past the last page are -1
 *   len    [max_seqs] tokens of each sequence
 * An empty cache has ref = 0, table = -1, len = 0.  A partly filled last page
 * belongs to one sequence (the calls below keep it so), so appending never
 * writes to a shared page.  dtype XC_F32 / XC_BF16; head_dim 16, 32, 64 or
 * 128 (the attention reads XC_BF16 caches of 64 and 128); page_size a power of
 * two from 16 to 1024; n_pages * page_size < 2^31.
 * Calls on one cache must be ordered (one stream, or events).
 *
 * What the host cannot see is checked on the device: a call that finds a bad
 * value sets a bit of the word xc_op_device_error() returns --
 * XC_DEV_CACHE_FULL or XC_DEV_BAD_SEQUENCE for the page calls, of which fork
 * and extend then change nothing; XC_DEV_BAD_POSITION for a position or slot out of range,
 * whose token is then skipped.  The first operator call of a process sets up
 * that word; it should come before any stream capture. */
typedef struct {
    int dtype, n_layers, n_pages, page_size, n_kv_heads, head_dim, max_seqs, max_pages;
    void *k, *v;
    int *ref, *table, *len;
} xc_kv_cache;

enum {
    XC_DEV_CACHE_FULL = 64,      /* not enough free pages, or a full table row */
    XC_DEV_BAD_SEQUENCE = 128,   /* sequence id, length or page id out of range; a fork into
                                    a sequence that is not empty; a sequence listed twice */
    XC_DEV_BAD_POSITION = 256    /* rotation position or cache slot out of range */
};

/* Bytes of device workspace of xc_op_kv_fork / _extend / _compact on this
 * cache (page lists).  Contents on entry are ignored. */
size_t xc_op_kv_workspace_bytes(const xc_kv_cache *cache);

/* For i < n (n <= 1024): sequence dst[i] (empty) becomes a copy of src[i]
 * (device int arrays; a sequence may be forked to many).  Full pages are shared (ref + 1);
 * the rows in use of a partly filled last page are copied, in every layer,
 * into a fresh page: the lowest free page ids, in list order. */
xc_status xc_op_kv_fork(const xc_kv_cache *cache, int n, const int *src, const int *dst, void *workspace,
                        size_t workspace_bytes, void *stream);

/* Appends n_new tokens to each of the n <= 1024 listed sequences: takes the pages they
 * need (lowest free ids first, in list order, then token order), advances len
 * and writes the cache slot of every new token, page * page_size + offset, to
 * slots [n][n_new] (-1 everywhere when the call changes nothing). */
xc_status xc_op_kv_extend(const xc_kv_cache *cache, int n, const int *seqs, int n_new, int *slots,
                          void *workspace, size_t workspace_bytes, void *stream);

/* Empties the n listed sequences: ref - 1 of their pages, table entries -1,
 * len 0.  An empty sequence stays as it is.  An id out of range is flagged and
 * skipped; the others are emptied. */
xc_status xc_op_kv_free(const xc_kv_cache *cache, int n, const int *seqs, void *stream);

/* Moves the pages in use to ids 0 .. n_live - 1: the k-th page in use with an
 * id >= n_live goes to the k-th free id below n_live (both ascending), in
 * every layer; ref and table follow.  *n_live (device) receives the count.
 * The contents of pages that become free are left as they are. */
xc_status xc_op_kv_compact(const xc_kv_cache *cache, int *n_live, void *workspace, size_t workspace_bytes,
                           void *stream);

/* Rotation table: for each axis a of n_axes (1 to 4), positions 0 ..
 * n_pos[a] - 1 and pairs 0 .. axis_pairs[a] - 1 (host arrays), (cos, sin) of
 * position * theta^(-pair / axis_pairs[a]), as float pairs
 * [n_pos[a]][axis_pairs[a]][2], axis after axis, computed in double. */
xc_status xc_op_rope_table(int n_axes, const int *axis_pairs, const int *n_pos, double theta, float *table,
                           void *stream);

/* Head-wise RMS norm of queries and keys, position rotation and the write into
 * the cache, in one pass.  For token t and head h, y = x / sqrt(mean(x^2) +
 * eps) * gamma (gamma_q / gamma_k float [head_dim]), then pair p of y rotates
 * by the table entry of the token's position on the pair's axis (axes own
 * consecutive pairs, axis_pairs[a] each, head_dim / 2 in all): (a, b) -> (a cos -
 * b sin, a sin + b cos), a pair being elements (2p, 2p + 1), or with
 * half_split (p, p + head_dim / 2).  Queries go to q_out, keys and the
 * unchanged values to row slots[t] of this layer's pages; slots[t] = -1 keeps
 * no keys of the token.  Rounded once, at the store.
 *   q, q_out  [n_tokens][n_heads * head_dim], rows q_stride / q_out_stride
 *             elements apart; q_out may be q itself
 *   k, v      [n_tokens][n_kv_heads * head_dim], rows k_stride / v_stride apart
 *   pos       device int [n_tokens][n_axes], 0 <= pos < n_pos[axis]
 *   slots     device int [n_tokens], distinct except for -1
 * Rows are 16-byte aligned.  n_heads is a multiple of the cache's n_kv_heads. */
xc_status xc_op_qk_norm_rope(const xc_kv_cache *cache, int layer, int n_tokens, int n_heads, const void *q,
                             long q_stride, const void *k, long k_stride, const void *v, long v_stride,
                             const float *gamma_q, const float *gamma_k, float eps, int n_axes,
                             const int *axis_pairs, const int *n_pos, const int *pos, const float *table,
                             int half_split, const int *slots, void *q_out, long q_out_stride, void *stream);

/* Attention of a batch of branches over one layer of the cache.  Query row
 * t = b * n_q + i (b < n_branches, i < n_q) belongs to sequence seqs[b]; head h
 * reads key head h / (n_heads / n_kv_heads):
 *   o[t] = sum_j p_j v_j, p = softmax over j < limit of scale * (q[t] . k_j),
 * limit = len (causal = 0), or with causal = 1 len - n_q + i + 1: the queries
 * are the sequence's last n_q tokens.  A row that sees no key gives 0.
 *   shared_len  the first shared_len tokens (a multiple of page_size) of every
 *               listed sequence are the same pages, as after a fork: they are
 *               read once for all branches, from the row of seqs[0].  Which
 *               keys a row sees does not depend on it.  Keys and values
 *               behind a page id out of range, or in the row of a seqs[0]
 *               out of range, count as 0, and the call is flagged.
 *   scale       > 0, or 0 for 1 / sqrt(head_dim)
 *   q, o        [n_branches * n_q][n_heads * head_dim], rows q_stride / o_stride
 *               elements apart, 16-byte aligned
 *   workspace   device, at least xc_op_branch_attention_workspace_bytes();
 *               contents on entry are ignored; not shared by overlapping calls
 * Cache rows that no sequence has reached (the rest of a last page) may hold
 * anything.  A key that the causal limit hides from a row but that is part of
 * the sequence must be finite, as must its value.  XC_BF16 needs head_dim 64
 * or 128.  At most 128 query heads per key head (XC_F32: 64).  Every branch has
 * n_q new tokens, and only one common part is read once: the children of two
 * parents read each parent's pages once a branch.
 * Scores, maxima, sums and partial results are fp32.  For XC_BF16 the weights
 * p_j are rounded to bf16 for the product with v, and the output once: rel-L2
 * 2.3e-3 against 64 bits on long sequences, where rounding the exact output
 * alone gives 1.7e-3.  XC_F32 rounds nothing to fewer bits.
 * A call is refused when the line of key tiles would not fit 32 bits with every
 * table row full, since the lengths are the device's and may have grown when a
 * captured call is replayed. */
size_t xc_op_branch_attention_workspace_bytes(const xc_kv_cache *cache, int n_branches, int n_q, int n_heads,
                                              int shared_len);
xc_status xc_op_branch_attention(const xc_kv_cache *cache, int layer, int n_branches, const int *seqs, int n_q,
                                 int n_heads, const void *q, long q_stride, int shared_len, int causal,
                                 float scale, void *o, long o_stride, void *workspace, size_t workspace_bytes,
                                 void *stream);

/* 1 while work given to `stream` is captured into a graph, else 0.  A captured
 * call uses its pointers again at every replay: its workspace must live as long
 * as the graph, and must not be shared with calls that overlap a replay. */
int xc_op_stream_capturing(void *stream);

/* Reads and clears the process-wide device error word of operator calls
 * (synchronising).  0 = no error. */
int xc_op_device_error(void);

#ifdef __cplusplus
}
#endif
#endif /* XCACHE_OPS_H */
