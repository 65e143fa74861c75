/* Residual addition with dropout on one MI355X (gfx950): the step between the
 * pair stack's operators (z += dropout(update)), with a mask that is never
 * stored.  For the pair (i, j) and channel c of a [rows][cols][channels] tensor
 *
 *     out_ijc = res_ijc + (kept_ijc ? x_ijc / (1 - p) : 0)
 *     dx_ijc  =           (kept_ijc ? dout_ijc / (1 - p) : 0)
 *
 * (the gradient of res is dout itself).  kept is a function of the seed, the
 * offset and the element alone, so the backward and every device of a 2-D grid
 * of tiles find the same mask without exchanging it: with r = row0 + i and
 * s = col0 + j, the element's place in the whole tensor,
 *
 *     e = (r * n_cols + s) * channels + c,  r = 0 when the rows share a mask,
 *                                           s = 0 when the columns do,
 *     kept = word (e % 4) of Philox-4x32-10(counter = (e / 4, offset), key = seed) >= round(p 2^32)
 *
 * (Salmon, Moraes, Dror and Shaw, SC 2011; counter words from the low to the
 * high: e / 4 in two, offset in two; key the seed's low and high word).
 * Sharing: the row-wise and column-wise dropout of the pair stack drop a
 * channel for a whole row or column of pairs.
 *
 * A dropped x is not looked at (NaN included).  out may be res or x itself, dx
 * may be dout itself, where types and strides agree.  Arithmetic in fp32, one
 * rounding.  Conventions as in tri_mul.h: device pointers, status codes
 * TRI_MUL_*, message in tri_mul_last_error(), asynchronous on `stream`, no
 * workspace, capturable.  seed and offset are values of the call: each replay
 * of a captured one drops the same elements, so a training step that is captured
 * is captured again for another mask.
 */
#ifndef PAIR_DROPOUT_H
#define PAIR_DROPOUT_H

#include <stdint.h>

#include "tri_mul.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { PAIR_DROPOUT_EACH = 0, PAIR_DROPOUT_ROWS = 1, PAIR_DROPOUT_COLUMNS = 2 };

typedef struct {
    int64_t rows, cols, channels;   /* this call's tile; any may be 0                                  */
    int64_t row0, col0, n_cols;     /* its place in the whole tensor, and that tensor's columns        */
    int64_t ld_x, ld_out;           /* elements from one row to the next: x (dx); res, out (dout)      */
    int32_t x_dtype, out_dtype;     /* TRI_MUL_F32 or TRI_MUL_BF16: x, dx; res, out, dout              */
    int32_t share;                  /* PAIR_DROPOUT_EACH: a mask value per element; _ROWS: all rows have
                                       the same mask; _COLUMNS: all columns have                       */
    double p;                       /* probability of dropping, [0, 1)                                 */
    uint64_t seed, offset;          /* a training step's own, and for instance the layer's             */
} pair_dropout_view_t;

/* res: as out, or NULL for 0.  Pairs and channels are contiguous within a row;
 * pointers need only their type's alignment (16-byte alignment, row strides to
 * match and a multiple of 8 channels are fastest).  Errors: EINVAL for null or
 * misaligned pointers, sizes, row strides below cols * channels, a tile outside
 * the columns, p, types or sharing outside their range; EUNSUPPORTED for a
 * tensor of 2^62 elements or a row of 2^31; EHIP for a failed launch. */
int pair_dropout_add(const pair_dropout_view_t* v, const void* x, const void* res, void* out, void* stream);

/* dx from dout with the mask of the pair_dropout_add of the same view. */
int pair_dropout_backward(const pair_dropout_view_t* v, const void* dout, void* dx, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PAIR_DROPOUT_H */
