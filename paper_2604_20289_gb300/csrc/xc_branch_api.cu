// Operator entry points of branched rollouts (include/xcache_ops.h): argument
// checks on the host, then the launches.  What only the device can see (the
// page state, positions) is checked by the kernels.
#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "xc_branch.cuh"
#include "xc_kernels.cuh"

using namespace xc;

int xc::device_sms() {
    static int n = 0;
    if (n == 0) {
        int dev = 0, x = 0;
        cudaGetDevice(&dev);
        if (cudaDeviceGetAttribute(&x, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || x < 1) return 1;
        n = x;
    }
    return n;
}

namespace {

xc_status fail(xc_status st, const char *fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    set_global_error(msg);
    return st;
}
xc_status launched(const char *what, cudaError_t e) {
    if (e == cudaSuccess) return XC_OK;
    return fail(e == cudaErrorInvalidValue ? XC_EINVAL : XC_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// Rows of `cols` elements, `ld` apart, each 16-byte aligned.
bool rows_ok(const void *p, long ld, long cols, int dtype) {
    return p != nullptr && aligned16(p) && ld >= cols && ld < (1l << 36) && (ld * (long)elem_bytes(dtype)) % 16 == 0;
}

bool cache_shape_ok(const xc_kv_cache *c) {
    return c != nullptr && (c->dtype == XC_F32 || c->dtype == XC_BF16) && c->n_layers >= 1 && c->n_pages >= 1 &&
           c->page_size >= 16 && c->page_size <= 1024 && (c->page_size & (c->page_size - 1)) == 0 &&
           c->n_kv_heads >= 1 && c->n_kv_heads <= 4096 &&
           (c->head_dim == 16 || c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 128) && c->max_seqs >= 1 &&
           c->max_pages >= 1 && (long long)c->n_pages * c->page_size < (1ll << 31) &&
           (long long)c->max_pages * c->page_size < (1ll << 30);
}
xc_status check_cache(const char *who, const xc_kv_cache *c) {
    if (!cache_shape_ok(c))
        return fail(XC_EINVAL, "%s: cache: dtype f32 / bf16, head_dim 16 / 32 / 64 / 128, page_size a power of two in "
                               "[16, 1024], positive counts, n_pages * page_size < 2^31", who);
    if (c->k == nullptr || c->v == nullptr || c->ref == nullptr || c->table == nullptr || c->len == nullptr ||
        !aligned16(c->k) || !aligned16(c->v))
        return fail(XC_EINVAL, "%s: cache: NULL or unaligned pointer", who);
    return XC_OK;
}
xc_status check_ws(const char *who, const void *ws, size_t have, size_t need) {
    if (ws == nullptr || !aligned16(ws) || have < need)
        return fail(XC_EINVAL, "%s: workspace of %zu bytes needed (16-byte aligned)", who, need);
    return XC_OK;
}
xc_status check_axes(const char *who, int n_axes, const int *pairs, const int *n_pos, RopeAxes *ax, long *sum) {
    if (n_axes < 1 || n_axes > ROPE_AXES || pairs == nullptr || n_pos == nullptr)
        return fail(XC_EINVAL, "%s: 1 to %d position axes", who, ROPE_AXES);
    *ax = RopeAxes{};
    ax->n = n_axes;
    *sum = 0;
    long long entries = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (pairs[a] < 1 || pairs[a] > 512 || n_pos[a] < 1) return fail(XC_EINVAL, "%s: empty position axis", who);
        ax->pairs[a] = pairs[a];
        ax->n_pos[a] = n_pos[a];
        *sum += pairs[a];
        entries += (long long)pairs[a] * n_pos[a];
    }
    if (entries >= (1ll << 31)) return fail(XC_EINVAL, "%s: rotation table too large", who);
    return XC_OK;
}
#define CHECK(call)                          \
    do {                                     \
        const xc_status s_ = (call);         \
        if (s_ != XC_OK) return s_;          \
    } while (0)
#define ERR_WORD(err, who)                                     \
    int *err = op_error_word();                                \
    if (err == nullptr) return fail(XC_ECUDA, who ": error word")
cudaStream_t as_stream(void *s) { return reinterpret_cast<cudaStream_t>(s); }

}  // namespace

extern "C" {

size_t xc_op_kv_workspace_bytes(const xc_kv_cache *cache) {
    return cache_shape_ok(cache) ? kv_workspace_bytes(*cache) : 0;
}

xc_status xc_op_kv_fork(const xc_kv_cache *cache, int n, const int *src, const int *dst, void *workspace,
                        size_t workspace_bytes, void *stream) {
    CHECK(check_cache("xc_op_kv_fork", cache));
    if (n < 0 || n > cache->max_seqs || n > KV_LIST_MAX || (n > 0 && (src == nullptr || dst == nullptr)))
        return fail(XC_EINVAL, "xc_op_kv_fork: 0 to max_seqs, and to %d, pairs of sequences", KV_LIST_MAX);
    if (n == 0) return XC_OK;
    CHECK(check_ws("xc_op_kv_fork", workspace, workspace_bytes, kv_workspace_bytes(*cache)));
    ERR_WORD(err, "xc_op_kv_fork");
    return launched("xc_op_kv_fork", kv_fork(*cache, n, src, dst, workspace, err, as_stream(stream)));
}

xc_status xc_op_kv_extend(const xc_kv_cache *cache, int n, const int *seqs, int n_new, int *slots,
                          void *workspace, size_t workspace_bytes, void *stream) {
    CHECK(check_cache("xc_op_kv_extend", cache));
    if (n < 0 || n > cache->max_seqs || n > KV_LIST_MAX || n_new < 0 || n_new > cache->max_pages * cache->page_size ||
        (n > 0 && n_new > 0 && (seqs == nullptr || slots == nullptr)))
        return fail(XC_EINVAL, "xc_op_kv_extend: 0 to max_seqs, and to %d, sequences, n_new up to a table row", KV_LIST_MAX);
    if (n == 0 || n_new == 0) return XC_OK;
    CHECK(check_ws("xc_op_kv_extend", workspace, workspace_bytes, kv_workspace_bytes(*cache)));
    ERR_WORD(err, "xc_op_kv_extend");
    return launched("xc_op_kv_extend", kv_extend(*cache, n, seqs, n_new, slots, workspace, err, as_stream(stream)));
}

xc_status xc_op_kv_free(const xc_kv_cache *cache, int n, const int *seqs, void *stream) {
    CHECK(check_cache("xc_op_kv_free", cache));
    if (n < 0 || (n > 0 && seqs == nullptr)) return fail(XC_EINVAL, "xc_op_kv_free: bad list");
    if (n == 0) return XC_OK;
    ERR_WORD(err, "xc_op_kv_free");
    return launched("xc_op_kv_free", kv_free(*cache, n, seqs, err, as_stream(stream)));
}

xc_status xc_op_kv_compact(const xc_kv_cache *cache, int *n_live, void *workspace, size_t workspace_bytes,
                           void *stream) {
    CHECK(check_cache("xc_op_kv_compact", cache));
    if (n_live == nullptr) return fail(XC_EINVAL, "xc_op_kv_compact: n_live is NULL");
    CHECK(check_ws("xc_op_kv_compact", workspace, workspace_bytes, kv_workspace_bytes(*cache)));
    return launched("xc_op_kv_compact", kv_compact(*cache, n_live, workspace, as_stream(stream)));
}

xc_status xc_op_rope_table(int n_axes, const int *axis_pairs, const int *n_pos, double theta, float *table,
                           void *stream) {
    RopeAxes ax;
    long sum = 0;
    CHECK(check_axes("xc_op_rope_table", n_axes, axis_pairs, n_pos, &ax, &sum));
    if (!(theta > 0.0) || !std::isfinite(theta) || table == nullptr || (reinterpret_cast<uintptr_t>(table) & 7) != 0)
        return fail(XC_EINVAL, "xc_op_rope_table: theta > 0 and an 8-byte aligned table");
    return launched("xc_op_rope_table", rope_axes_table(ax, theta, reinterpret_cast<float2 *>(table), as_stream(stream)));
}

xc_status xc_op_qk_norm_rope(const xc_kv_cache *cache, int layer, int n_tokens, int n_heads, const void *q,
                             long q_stride, const void *k, long k_stride, const void *v, long v_stride,
                             const float *gamma_q, const float *gamma_k, float eps, int n_axes,
                             const int *axis_pairs, const int *n_pos, const int *pos, const float *table,
                             int half_split, const int *slots, void *q_out, long q_out_stride, void *stream) {
    const char *who = "xc_op_qk_norm_rope";
    CHECK(check_cache(who, cache));
    const xc_kv_cache &c = *cache;
    if (layer < 0 || layer >= c.n_layers || n_tokens < 0) return fail(XC_EINVAL, "%s: layer or token count", who);
    if (n_heads < 1 || n_heads % c.n_kv_heads != 0 || n_heads > 65536)
        return fail(XC_EINVAL, "%s: n_heads must be a multiple of the cache's n_kv_heads", who);
    if ((long long)n_tokens * (n_heads + 2 * c.n_kv_heads) >= (1ll << 31))
        return fail(XC_EINVAL, "%s: too many token rows", who);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(XC_EINVAL, "%s: eps", who);
    NormRopeArgs a{};
    long sum = 0;
    CHECK(check_axes(who, n_axes, axis_pairs, n_pos, &a.ax, &sum));
    if (sum != c.head_dim / 2) return fail(XC_EINVAL, "%s: axis_pairs must add up to head_dim / 2", who);
    if (n_tokens == 0) return XC_OK;
    const long dq = (long)n_heads * c.head_dim, dk = (long)c.n_kv_heads * c.head_dim;
    if (!rows_ok(q, q_stride, dq, c.dtype) || !rows_ok(k, k_stride, dk, c.dtype) || !rows_ok(v, v_stride, dk, c.dtype) ||
        !rows_ok(q_out, q_out_stride, dq, c.dtype))
        return fail(XC_EINVAL, "%s: rows must be 16-byte aligned and at least as far apart as they are wide", who);
    if (gamma_q == nullptr || gamma_k == nullptr || !aligned16(gamma_q) || !aligned16(gamma_k) || pos == nullptr ||
        table == nullptr || (reinterpret_cast<uintptr_t>(table) & 7) != 0 || slots == nullptr)
        return fail(XC_EINVAL, "%s: NULL or unaligned pointer", who);
    ERR_WORD(err, "xc_op_qk_norm_rope");
    a.T = n_tokens;
    a.H = n_heads;
    a.Hk = c.n_kv_heads;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_ld = q_stride;
    a.k_ld = k_stride;
    a.v_ld = v_stride;
    a.o_ld = q_out_stride;
    a.gamma_q = gamma_q;
    a.gamma_k = gamma_k;
    a.eps = eps;
    a.pos = pos;
    a.table = reinterpret_cast<const float2 *>(table);
    a.slots = slots;
    a.q_out = q_out;
    a.n_rows = (long)c.n_pages * c.page_size;
    const size_t layer_off = (size_t)layer * a.n_rows * kv_row_bytes(c);
    a.k_pool = reinterpret_cast<char *>(c.k) + layer_off;
    a.v_pool = reinterpret_cast<char *>(c.v) + layer_off;
    a.err = err;
    return launched(who, qk_norm_rope(c.dtype, c.head_dim, half_split != 0, a, as_stream(stream)));
}

static xc_status check_branch(const char *who, const xc_kv_cache *cache, int n_branches, int n_q, int n_heads,
                              int shared_len) {
    if (!cache_shape_ok(cache)) return check_cache(who, cache);
    const xc_kv_cache &c = *cache;
    if (n_branches < 0 || n_q < 0 || (long long)n_branches * n_q >= (1ll << 31))
        return fail(XC_EINVAL, "%s: n_branches, n_q", who);
    if (n_heads < 1 || n_heads % c.n_kv_heads != 0 || n_heads / c.n_kv_heads > (c.dtype == XC_F32 ? 64 : 128))
        return fail(XC_EINVAL, "%s: n_heads must be a multiple of the cache's n_kv_heads, up to 128 (f32: 64) times it", who);
    if (c.dtype == XC_BF16 && c.head_dim < 64) return fail(XC_EINVAL, "%s: bf16 needs head_dim 64 or 128", who);
    if (shared_len < 0 || shared_len % c.page_size != 0 || shared_len > c.max_pages * c.page_size)
        return fail(XC_EINVAL, "%s: shared_len must be a multiple of page_size within a table row", who);
    if (n_branches > 0 && n_q > 0 && ((long long)n_branches * n_q * n_heads >= (1ll << 31) ||
                                      !branch_attn_fits(c, n_branches, n_q, n_heads, shared_len)))
        return fail(XC_EINVAL, "%s: too many query rows for tables this long", who);
    return XC_OK;
}

size_t xc_op_branch_attention_workspace_bytes(const xc_kv_cache *cache, int n_branches, int n_q, int n_heads,
                                              int shared_len) {
    if (check_branch("xc_op_branch_attention_workspace_bytes", cache, n_branches, n_q, n_heads, shared_len) != XC_OK)
        return 0;
    if (n_branches == 0 || n_q == 0) return 0;
    return branch_attn_workspace_bytes(*cache, n_branches, n_q, n_heads, shared_len);
}

xc_status xc_op_branch_attention(const xc_kv_cache *cache, int layer, int n_branches, const int *seqs, int n_q,
                                 int n_heads, const void *q, long q_stride, int shared_len, int causal,
                                 float scale, void *o, long o_stride, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    const char *who = "xc_op_branch_attention";
    CHECK(check_cache(who, cache));
    const xc_kv_cache &c = *cache;
    if (layer < 0 || layer >= c.n_layers) return fail(XC_EINVAL, "%s: layer", who);
    CHECK(check_branch(who, cache, n_branches, n_q, n_heads, shared_len));
    if (!(scale >= 0.0f) || !std::isfinite(scale)) return fail(XC_EINVAL, "%s: scale must be finite and not negative", who);
    if (n_branches == 0 || n_q == 0) return XC_OK;
    const long d = (long)n_heads * c.head_dim;
    if (!rows_ok(q, q_stride, d, c.dtype) || !rows_ok(o, o_stride, d, c.dtype))
        return fail(XC_EINVAL, "%s: rows must be 16-byte aligned and at least as far apart as they are wide", who);
    if (seqs == nullptr) return fail(XC_EINVAL, "%s: seqs is NULL", who);
    CHECK(check_ws(who, workspace, workspace_bytes, branch_attn_workspace_bytes(c, n_branches, n_q, n_heads, shared_len)));
    ERR_WORD(err, "xc_op_branch_attention");
    BranchAttnArgs a{};
    a.B = n_branches;
    a.n_q = n_q;
    a.H = n_heads;
    a.Hk = c.n_kv_heads;
    a.shared = shared_len;
    a.causal = causal != 0;
    a.scale = scale > 0.0f ? scale : 1.0f / sqrtf((float)c.head_dim);
    a.seqs = seqs;
    a.q = q;
    a.q_ld = q_stride;
    a.o = o;
    a.o_ld = o_stride;
    const size_t layer_off = (size_t)layer * c.n_pages * c.page_size * kv_row_bytes(c);
    a.k = reinterpret_cast<const char *>(c.k) + layer_off;
    a.v = reinterpret_cast<const char *>(c.v) + layer_off;
    return launched(who, branch_attn(c, a, workspace, err, as_stream(stream)));
}

int xc_op_stream_capturing(void *stream) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    if (stream == nullptr) return 0;                       // the legacy default stream is never captured
    if (cudaStreamIsCapturing(as_stream(stream), &status) != cudaSuccess) {
        cudaGetLastError();                                // cleared: the stream's next call reports it
        return 0;
    }
    return status != cudaStreamCaptureStatusNone;
}

}  // extern "C"
