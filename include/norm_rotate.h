/* Norms of queries and keys for each head with the position rotation in the same
 * pass, on one MI355X (gfx950): what stands between the projections and the
 * attention of cross_attn.h, with its gradients.
 *
 * For a head's row x of d values, of the token at position p:
 *
 *     layer = 0:  r = 1 / sqrt(mean(x^2) + eps),           u = x r
 *     layer = 1:  r = 1 / sqrt(mean((x - mu)^2) + eps),    u = (x - mu) r,  mu = mean(x)
 *     w = u gain + shift
 *     y_a = w_a cos(p f_m) - w_b sin(p f_m),  y_b = w_a sin(p f_m) + w_b cos(p f_m)
 *
 * for the pairs m < rot / 2 of the first rot values -- (a, b) = (m, m + rot / 2), or
 * (2m, 2m + 1) with adjacent = 1 -- and y = w behind them.  With g the gradient of y
 * turned back and h = g gain:
 *
 *     dgain = sum of g u,  dshift = sum of g  (over all rows of the queries, or of the keys)
 *     dx = r (h - u mean(h u))            less r mean(h) where layer = 1
 *
 * Queries and keys are two sides of one call, with their own heads and weights and
 * the same tokens; a side may be missing (NULL), as for queries and keys of
 * different lengths, which take a call each.  The gradient needs x; the forward can
 * leave it in 8 bits (checkpoint8.h, a group for each row), and the backward takes
 * that in the place of x: its u and r are those of the values it stands for.
 *
 * Conventions as in cross_attn.h: tensors [batch][n][heads][d] of `dtype` with unit
 * stride along d, 16-byte aligned data and strides that are multiples of 16 bytes (a
 * stride of 0 repeats an input); device pointers, status codes, message in
 * tri_mul_last_error(), asynchronous on `stream`, capturable.  y may be x, and dx may be
 * dy or x, where strides agree; otherwise no output may overlap an input.  Rows are
 * independent: NaN or infinities show in their own row (and in dgain and dshift, which
 * sum over all rows: the dy of padding has to be 0 and its x finite).  Squares, sums and
 * weights' gradients in fp32 and wider, in a fixed order; angles in 64 bits; one
 * rounding of y and dx.  A row whose squares pass fp32's range (values from about
 * 10^18 on) has u and r of 0, or NaN where its sum passes it too.
 */
#ifndef NORM_ROTATE_H
#define NORM_ROTATE_H

#include <stddef.h>
#include <stdint.h>

#include "cross_attn.h"
#include "tri_mul.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t batch, n;               /* entries and tokens of each; may be 0                               */
    int32_t d;                      /* a multiple of 8 in [8, 256]                                        */
    int32_t rot;                    /* a multiple of 8 in [0, d]                                          */
    int32_t dtype, weight_dtype;    /* TRI_MUL_F32 or TRI_MUL_BF16: x, y, dy, dx; gain, shift             */
    int32_t layer, adjacent;        /* 0 or 1                                                             */
    float eps;                      /* > 0                                                                */
    const int32_t* positions;       /* [n] of each entry (not looked at with rot = 0)                     */
    int64_t positions_batch;        /* from an entry's to the next's; 0: one for all                      */
    const double* freqs;            /* [rot / 2]: radians per position; angles below 2^50                 */
} norm_rotate_view_t;

/* The queries, or the keys. */
typedef struct {
    int32_t heads;                  /* in [1, 1024]                                                       */
    cross_attn_tensor_t x;          /* backward: data NULL to take codes and powers                       */
    const void *gain, *shift;       /* [d], or NULL for 1 and 0                                           */
    int8_t* codes;                  /* [batch][n][heads][d], 16-byte aligned; forward: written if not NULL */
    uint8_t* powers;                /* [batch][n][heads]                                                  */
} norm_rotate_side_t;

typedef struct {
    cross_attn_tensor_t dy, dx;
    float *dgain, *dshift;          /* [d] fp32, written whole; or NULL                                   */
} norm_rotate_grad_t;

/* yq and yk from the two sides (k and yk, or q and yq, may be NULL).  Errors: EINVAL
 * for null or misaligned pointers, sizes, strides, types, eps; EUNSUPPORTED for 2^31
 * entries or tokens, 2^44 values, strides of 2^40; EHIP for a failed launch. */
int norm_rotate_forward(const norm_rotate_view_t* v, const norm_rotate_side_t* q, const norm_rotate_side_t* k,
                        const cross_attn_tensor_t* yq, const cross_attn_tensor_t* yk, void* stream);

/* Bytes of the workspace of norm_rotate_backward (the partial sums of the weights' gradients). */
int norm_rotate_backward_workspace_size(const norm_rotate_view_t* v, const norm_rotate_side_t* q,
                                        const norm_rotate_side_t* k, size_t* bytes);

/* dx, dgain and dshift of the sides given, from x or from codes and powers (both sides
 * alike).  ws: 256-byte aligned (NULL if 0 bytes); ENOMEM for a small one. */
int norm_rotate_backward(const norm_rotate_view_t* v, const norm_rotate_side_t* q, const norm_rotate_side_t* k,
                         const norm_rotate_grad_t* gq, const norm_rotate_grad_t* gk, void* ws, size_t ws_bytes,
                         void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NORM_ROTATE_H */
