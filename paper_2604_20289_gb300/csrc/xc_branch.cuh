// Kernels of branched rollouts (k_kv_pages.cu, k_branch_attn.cu): the paged
// key / value cache and what fills, reorganises and reads it.
#pragma once
#include <cuda.h>

#include "xc_common.cuh"

namespace xc {

enum : int { ERR_CACHE_FULL = XC_DEV_CACHE_FULL, ERR_BAD_SEQ = XC_DEV_BAD_SEQUENCE, ERR_BAD_POS = XC_DEV_BAD_POSITION };

inline size_t elem_bytes(int dtype) { return dtype == XC_BF16 ? 2 : 4; }
inline size_t kv_row_bytes(const xc_kv_cache &c) { return (size_t)c.n_kv_heads * c.head_dim * elem_bytes(c.dtype); }

constexpr int KV_LIST_MAX = 1024;     // sequences of one fork or extend
size_t kv_workspace_bytes(const xc_kv_cache &c);
cudaError_t kv_fork(const xc_kv_cache &c, int n, const int *src, const int *dst, void *ws, int *err, cudaStream_t st);
cudaError_t kv_extend(const xc_kv_cache &c, int n, const int *seqs, int n_new, int *slots, void *ws, int *err,
                      cudaStream_t st);
cudaError_t kv_free(const xc_kv_cache &c, int n, const int *seqs, int *err, cudaStream_t st);
cudaError_t kv_compact(const xc_kv_cache &c, int *n_live, void *ws, cudaStream_t st);

constexpr int ROPE_AXES = 4;
struct RopeAxes {
    int n;
    int pairs[ROPE_AXES], n_pos[ROPE_AXES];
};
cudaError_t rope_axes_table(const RopeAxes &ax, double theta, float2 *out, cudaStream_t st);

struct NormRopeArgs {
    int T, H, Hk;
    const void *q, *k, *v;
    long q_ld, k_ld, v_ld, o_ld;      // row strides in elements
    const float *gamma_q, *gamma_k;
    float eps;
    RopeAxes ax;
    const int *pos;                   // [T][ax.n]
    const float2 *table;
    const int *slots;                 // [T]
    void *q_out, *k_pool, *v_pool;    // pools of the layer: rows of Hk * hd
    long n_rows;                      // rows of a layer's pool
    int *err;
};
cudaError_t qk_norm_rope(int dtype, int head_dim, bool half_split, const NormRopeArgs &a, cudaStream_t st);

struct BranchAttnArgs {
    int B, n_q, H, Hk, shared, causal;
    float scale;
    const int *seqs;
    const void *q;
    long q_ld, o_ld;
    void *o;
    const void *k, *v;                // the layer's pools
};
// Whether the line of key tiles fits the kernels' 32-bit counters.
bool branch_attn_fits(const xc_kv_cache &c, int B, int n_q, int H, int shared);
size_t branch_attn_workspace_bytes(const xc_kv_cache &c, int B, int n_q, int H, int shared);
cudaError_t branch_attn(const xc_kv_cache &c, const BranchAttnArgs &a, void *ws, int *err, cudaStream_t st);

// 3-D bf16 map of a [tokens][heads * head_dim] matrix (rows ld elements
// apart) with a box of 64 columns x box_heads heads x box_tokens tokens,
// 128-byte swizzle.
bool make_tmap_heads_bf16(CUtensorMap *m, const void *base, uint64_t head_dim, uint64_t heads, uint64_t tokens,
                          uint64_t ld, uint32_t box_heads, uint32_t box_tokens);
bool make_tmap_bf16(CUtensorMap *m, const void *base, uint64_t rows, uint64_t cols, uint32_t box_rows);
// Device error word of the operator entry points (NULL if it cannot be made).
int *op_error_word();
int device_sms();
}  // namespace xc
