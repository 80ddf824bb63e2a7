/* pp_act8.h -- C ABI of activations held in 8 bits, for AMD MI355X (gfx950).
 *
 * What a backward pass needs of a layer's input and output can wait for it in one byte a value.  For every
 * row of a matrix x [rows][n] and every block of 128 columns (the last block may be shorter), with
 * amax = max |x| over them:
 *
 *   e = the smallest whole number with amax <= 127 * 2^e, at least -126
 *   q = x / 2^e rounded to a whole number, ties to even, but +1 or -1 where that is 0 and x is not
 *   the value held is q * 2^e
 *
 * so a value is off by at most half of 2^e, by less than 2^e where it is below that, and its sign is never
 * lost: q > 0 says of a ReLU's output where the ReLU let through.  Dividing by a power of two is exact: the
 * held values are a function of x alone.  A block with an infinity or a NaN stands for NaN throughout (q keeps the signs,
 * +1 for a NaN).  Columns that stand for nothing, as a padded batch has them, count like any others: they are set to zero first.
 *
 * The buffer: q as int8 [rows][P], P = n rounded up to a multiple of 128, zeros behind n; then one byte e + 127
 * for each row and block (255: the block stands for NaN) as [P / 128][rows rounded up to a multiple of 16].
 * pp_adapter_grad_input and pp_adapter_grad_weights (pp_adapter.h) read it in this form.
 *
 * Pointers named *_dev are device pointers.  Status codes and dtypes are those of pp_conv.h.  No call throws,
 * synchronises or allocates.
 */
#ifndef PP_ACT8_H
#define PP_ACT8_H

#include <stdint.h>

#include "pp_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the buffer for a matrix of rows x n values; 0 if a size is < 1 or rows * n is beyond 2^31 - 1. */
int64_t pp_act8_bytes(int32_t rows, int32_t n);

/* Enqueue x [rows][n] (row-major, dtype) -> held_dev (pp_act8_bytes bytes).  Both 16-byte aligned and not overlapping
 * (PP_ERR_ALIGN otherwise).  PP_ERR_SHAPE: a size < 1, or rows * n beyond 2^31 - 1.  PP_ERR_UNSUPPORTED: an unknown dtype. */
pp_status_t pp_act8_pack(const void *x_dev, int32_t rows, int32_t n, int32_t dtype, void *held_dev, void *hip_stream);

/* Enqueue the values held, as x_dev [rows][n] of dtype.  A value beyond dtype's largest number, which in the dtype that was packed only
 * an x above 127 / 128 of it leads to, becomes that number, of its sign.  Same refusals. */
pp_status_t pp_act8_unpack(const void *held_dev, int32_t rows, int32_t n, int32_t dtype, void *x_dev, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* PP_ACT8_H */
