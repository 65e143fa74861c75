/* Activations held in 8 bits between forward and backward on one MI355X
 * (gfx950): about half of bf16's memory, a quarter of fp32's.
 *
 * A row of n values is cut into groups of `group` values (the last one may be
 * shorter).  A group holds one power of two and a signed byte for each value:
 *
 *     amax = the largest magnitude = m 2^e, 1 <= m < 2
 *     k    = e - 6 + (64 m rounds to more than 127 ? 1 : 0), within [-127, 121]
 *     code = x 2^-k rounded to the nearest whole number, halves to even, within [-127, 127]
 *     byte = k + 127                                 value = code 2^k
 *
 * (a group of zeros: code 0, byte 0; with an infinity or a NaN among its values:
 * byte 255, and the whole group reads back as NaN).  The scale is a power of two
 * so that x 2^-k is exact and a code has one value whoever computes it; a value
 * has 7 significant bits, so reading it back as bf16 or fp32 is exact too.  The
 * error is at most half a step, 2^(k-1), and that at most amax / 127 (amax / 254 at
 * best) except at the ends of k's range: groups whose amax is below 127 2^-128 are
 * held at k = -127 and are off by up to 2^-128 (from an amax of 2^-128 down by the
 * values themselves: all codes are 0), and where k would be 122 the error is a step
 * at most, so that no finite value reads back as infinity.
 *
 * norm_rotate.h writes this form in its forward pass (a group for each head's
 * row) and reads it in its backward.
 *
 * Conventions as in tri_mul.h: device pointers, status codes TRI_MUL_*, message
 * in tri_mul_last_error(), asynchronous on `stream`, no workspace, capturable.
 * No output may overlap an input.
 */
#ifndef CHECKPOINT8_H
#define CHECKPOINT8_H

#include <stdint.h>

#include "tri_mul.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t rows, n;     /* rows of n values; either may be 0                                         */
    int64_t ld;          /* elements from one row of x (out) to the next (not looked at with one row) */
    int32_t dtype;       /* TRI_MUL_F32 or TRI_MUL_BF16: x, out                                       */
    int32_t group;       /* a multiple of 8 in [8, 256]                                               */
} checkpoint8_view_t;

/* codes [rows][n] and powers [rows][ceil(n / group)] from x.  x needs only its
 * type's alignment, codes none (16-byte alignment of x, 8-byte of codes, and n
 * and ld multiples of 8 are fastest).  Errors: EINVAL for null or misaligned
 * pointers, sizes, ld below n, dtype or group outside their range; EUNSUPPORTED
 * for 2^40 rows, n or ld, or 2^62 values; EHIP for a failed launch. */
int checkpoint8_pack(const checkpoint8_view_t* v, const void* x, int8_t* codes, uint8_t* powers, void* stream);

/* The values that codes and powers stand for. */
int checkpoint8_unpack(const checkpoint8_view_t* v, const int8_t* codes, const uint8_t* powers, void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CHECKPOINT8_H */
