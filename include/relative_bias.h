/* Learned relative position bias by buckets on one MI355X (gfx950), with its
 * gradient: as the bias of cross_attn.h, and as the relative position encoding
 * of the pair tensor.
 *
 * A table holds a row for each bucket.  For query i at position p_i and key j at
 * position p_j
 *
 *     b_ij = buckets - 1                                     if segments are given and s_i != s_j,
 *            lut[min(max(p_j - p_i, -reach), reach) + reach]  otherwise
 *
 *     bias:  out_bhij = base_bhij + table[b_ij][h]     dtable[t][h] = sum of dout_bhij over b_ij = t
 *     pair:  out_ijc  = base_ijc  + table[b_ij][c]     dtable[t][c] = sum of dout_ijc  over b_ij = t
 *
 * (the gradient of base is dout itself).  Positions and segments (chains) are
 * any 32-bit integers, in any order; p_j - p_i does not overflow.  An entry of
 * lut that is not below `buckets` is taken as buckets - 1.
 *
 * Conventions as in tri_mul.h: device pointers, status codes TRI_MUL_*, message
 * in tri_mul_last_error(), asynchronous on `stream`, capturable (no allocation,
 * no memset), nothing kept between calls.  Sums in fp32 and wider, in a fixed
 * order: equal calls give equal bits.  One rounding of base + table.  out may be
 * base itself where strides agree; otherwise no output may overlap an input.
 */
#ifndef RELATIVE_BIAS_H
#define RELATIVE_BIAS_H

#include <stddef.h>
#include <stdint.h>

#include "cross_attn.h"
#include "tri_mul.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t batch, nq, nk;          /* entries, queries and keys of each (pair: 1, rows, columns); may be 0 */
    int32_t heads;                  /* columns of the table: heads, or channels of a pair; in [1, 1024]     */
    int32_t dtype, table_dtype;     /* TRI_MUL_F32 or TRI_MUL_BF16: base, out, dout; table                  */
    int32_t buckets;                /* rows of the table, in [1, 256]                                       */
    int32_t reach;                  /* in [0, 4095]                                                         */
    const uint8_t* lut;             /* [2 reach + 1]                                                        */
    const int32_t *pos_q, *pos_k;   /* [nq], [nk] of each entry                                             */
    int64_t pos_q_batch, pos_k_batch;   /* from an entry's to the next's; 0: one for all                    */
    const int32_t *seg_q, *seg_k;   /* both or neither                                                      */
    int64_t seg_q_batch, seg_k_batch;
} relative_view_t;

/* out [batch][heads][nq][nk] in the strides of a cross_attn_bias_t (a stride of 0
 * repeats base along batch or heads; out's are not 0 along axes longer than 1).
 * base: NULL for 0.  The values behind the nk-th of a row are neither read nor
 * written.  Data needs its type's alignment (16-byte alignment and strides that are
 * multiples of 8 are fastest).  Errors: EINVAL for null or misaligned pointers,
 * sizes, strides, types; EUNSUPPORTED for nq or nk of 2^24, 2^48 values, strides of 2^40 or more
 * than 2^24 - 1 work-groups; EHIP for a failed launch. */
int relative_bias(const relative_view_t* v, const void* table, const cross_attn_bias_t* base,
                  const cross_attn_bias_t* out, void* stream);

/* Bytes of the workspace of relative_bias_backward. */
int relative_bias_backward_workspace_size(const relative_view_t* v, size_t* bytes);

/* dtable [buckets][heads] fp32, written whole.  ws: 256-byte aligned (NULL if 0
 * bytes); ENOMEM for a small one. */
int relative_bias_backward(const relative_view_t* v, const cross_attn_bias_t* dout, float* dtable, void* ws,
                           size_t ws_bytes, void* stream);

/* out [nq][nk][heads] with rows ld_out elements apart; base (or NULL) likewise. */
int relative_pair(const relative_view_t* v, const void* table, const void* base, int64_t ld_base, void* out,
                  int64_t ld_out, void* stream);

int relative_pair_backward_workspace_size(const relative_view_t* v, size_t* bytes);

int relative_pair_backward(const relative_view_t* v, const void* dout, int64_t ld_dout, float* dtable, void* ws,
                           size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RELATIVE_BIAS_H */
