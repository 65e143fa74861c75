/* Attention of queries over keys of another length on one MI355X (gfx950):
 * cross attention to another sequence's states, attention with pair bias
 * (Fold-CP Section 3.6, Eq. 6), local windows, single queries over a long
 * sequence, and -- with the rows of a pair tensor as the batch and one bias for
 * all of them -- the triangle attention of triattn.h in a form that trains.
 *
 * For batch entry b, query i, head h and the key head hk = h / (heads / kv_heads):
 *
 *     x_ij  = scale q_bih . k_bj,hk + bias_bhij      over the keys j with mask_bj != 0
 *     out_bih = sum_j softmax_j(x_ij) v_bj,hk
 *
 * An absent key (mask 0) takes no part, whatever its k, v and bias hold (NaN
 * included).  A bias of -inf gives a key weight 0 for one query; its k and v are
 * multiplied all the same, so their products with q and dout have to be finite.
 * A query with no key left gives 0, and 0 gradients.  A finite bias is a number
 * like any other, the type's lowest value among them: a row that holds it
 * everywhere is the softmax of what fp32 keeps of the sum.
 *
 * Conventions shared with tri_mul.h: device pointers, status codes TRI_MUL_*,
 * message in tri_mul_last_error(), asynchronous on `stream` (a hipStream_t,
 * NULL = default stream) of the current device, validation before any launch.
 * Nothing is kept between calls: two calls may run at once on two streams with
 * two workspaces, and calls may be captured into graphs (no allocation, no
 * memset); graphs that replay at once need a workspace each.  All sums have a
 * fixed order: equal calls give equal bits.  No output may overlap an input.
 *
 * Tensors have `dtype` (TRI_MUL_F32 or TRI_MUL_BF16), unit stride along the
 * head's d values and the strides of cross_attn_tensor_t elsewhere; data is
 * 16-byte aligned and strides are multiples of 16 bytes.  A stride of 0 repeats
 * an input along that axis (batch and head; gradients cannot be written so).
 * Sizes: d a multiple of 8 in [8, 128]; heads in [1, 1024], a multiple of
 * kv_heads; batch, nq and nk may be 0; nq * heads / kv_heads and nk at most
 * 2^24; token strides below 2^23 elements.
 *
 * Precision: fp32 sums, softmax statistics and gradients throughout; with bf16
 * storage the softmax weights (and dS in the backward) enter their products
 * as bf16, an error of the size of the results' own rounding.  dout . out,
 * which the backward subtracts, is taken from out before its rounding (kept
 * beside the statistics): with few keys it is as large as what is left.
 */
#ifndef CROSS_ATTN_H
#define CROSS_ATTN_H

#include <stddef.h>
#include <stdint.h>

#include "tri_mul.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One [batch][tokens][heads][d] tensor; strides in elements. */
typedef struct {
    void* data;
    int64_t batch, token, head;
} cross_attn_tensor_t;

/* A bias, or its gradient: rows of nk values, `row` elements apart. */
typedef struct {
    void* data;                 /* 16-byte aligned; NULL: no bias                                     */
    int64_t batch, head;        /* from an entry's (head's) bias to the next's; 0: one for all        */
    int64_t row;                /* >= nk and at most 2^24; all three strides multiples of 8 (none is
                                   looked at along an axis of length 1)                               */
} cross_attn_bias_t;

typedef struct {
    int64_t batch, nq, nk;      /* entries, queries and keys of each                                  */
    int32_t heads, kv_heads;    /* heads of q and out; heads of k and v                               */
    int32_t d;                  /* channels of a head                                                 */
    int32_t dtype;              /* TRI_MUL_F32 or TRI_MUL_BF16: every tensor here but stats           */
    float scale;                /* > 0, usually 1 / sqrt(d)                                           */
    cross_attn_bias_t bias;     /* read up to the next multiple of 8 values behind nk                 */
    const uint8_t* mask;        /* [nk] bytes per entry, nonzero: key present; or NULL                */
    int64_t mask_batch;         /* from an entry's mask to the next's (bytes); 0: one for all         */
} cross_attn_view_t;

/* Bytes of the workspace of cross_attn_forward: the partial results of calls
 * that split the keys because there are few queries; 0 for the others. */
int cross_attn_workspace_size(const cross_attn_view_t* v, size_t* bytes);

/* Bytes of the stats that a forward leaves for its backward. */
int cross_attn_stats_size(const cross_attn_view_t* v, size_t* bytes);

/* out from q, k, vv (strides of each as given).  stats: NULL, or
 * cross_attn_stats_size bytes (16-byte aligned) for the backward: [2][batch][heads][nq]
 * fp32, each query's maximum of x, and its sum of exp(x - maximum) (-inf and 0 for
 * a query with no key); with bf16 storage also, from the next multiple of 256
 * bytes on, [batch][heads][nq][d] bf16, what the rounding took from out.  ws:
 * cross_attn_workspace_size bytes, 256-byte aligned (NULL if 0).  Errors:
 * EINVAL for null or misaligned pointers, bad sizes or strides; EUNSUPPORTED
 * for d, heads or sizes beyond the ones above; ENOMEM for a small workspace;
 * EHIP for a failed launch. */
int cross_attn_forward(const cross_attn_view_t* v, const cross_attn_tensor_t* q, const cross_attn_tensor_t* k,
                       const cross_attn_tensor_t* vv, const cross_attn_tensor_t* out, float* stats, void* ws,
                       size_t ws_bytes, void* stream);

/* Bytes of the workspace of cross_attn_backward (four fp32 values per query and
 * head, and the partial sums of dbias where few tiles of a bias are shared by
 * many entries or heads). */
int cross_attn_backward_workspace_size(const cross_attn_view_t* v, size_t* bytes);

/* Gradients for dout from the forward's out and stats.  dq, dk and dv are
 * written whole (the gradients of a key head summed over its query heads); dk
 * and dv may both be NULL (keys and values that do not learn).  dbias: NULL, or
 * the sums over the entries and heads that share a bias, with strides of its
 * own (ignored along an axis that v->bias shares); the values behind the nk-th
 * of its rows are left as they are. */
int cross_attn_backward(const cross_attn_view_t* v, const cross_attn_tensor_t* q, const cross_attn_tensor_t* k,
                        const cross_attn_tensor_t* vv, const cross_attn_tensor_t* out, const float* stats,
                        const cross_attn_tensor_t* dout, const cross_attn_tensor_t* dq,
                        const cross_attn_tensor_t* dk, const cross_attn_tensor_t* dv,
                        const cross_attn_bias_t* dbias, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CROSS_ATTN_H */
