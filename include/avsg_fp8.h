/* avsg_fp8.h — C ABI of matrices in 8-bit floating point with float32 scales, one
 * for each block of 128 columns: their quantisation and their product.  They serve
 * projections whose weights come in this form, beside the 4-bit ones of
 * avsg_latent.h.
 *
 * A code is e4m3 (the OCP form: one sign, four exponent and three mantissa bits, largest
 * value 448, no infinities); a value is its code times the scale of its block.  A
 * block is 128 columns of one row (activations) or 128 x 128 (weights); the last
 * block of a row, and the last rows of blocks, may be smaller.
 *
 * Conventions are those of avsg_latent.h: the caller owns all memory, the calls are
 * asynchronous on the given stream, allocate nothing, never throw or abort, can
 * be captured into a HIP graph and keep no state.  avsg_latent_last_error()
 * describes the calling thread's last failure.
 */
#ifndef AVSG_FP8_H
#define AVSG_FP8_H

#include "avsg_latent.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AVSG_FP8_BLOCK 128

/* A matrix, or a batch of them.  Codes are 16-byte aligned and their strides
 * multiples of 16; scales 4-byte aligned.  Row r, column c has the scale
 * d_scales[r / block_rows * scale_stride + c / 128]. */
typedef struct avsg_fp8 {
    const void *d_codes;
    const float *d_scales;
    int64_t code_stride, code_batch_stride;    /* bytes from row to row, from matrix to matrix */
    int64_t scale_stride, scale_batch_stride;  /* elements from a row of blocks to the next, from matrix to matrix */
    int32_t block_rows;                        /* 1 or 128 */
} avsg_fp8;

/* 8-bit form of x (AVSG_BF16 or AVSG_F32, [batch][rows][cols], rows 16-byte aligned,
 * strides in elements; cols a multiple of 16) into the codes and scales that `out` describes.
 * With a the largest magnitude of a block: code = x * (448 / a) rounded to the
 * nearest, ties to the even code, scale = a / 448, all in float32.  Below a = 2^-117 the
 * codes and the scale are zero; a block with an infinity or a NaN has scale NaN and codes
 * of zero.  batch is at most 65535, cols is below 2^31 - 128, and a matrix has at most 2^28 - 16
 * blocks of 1 x 128, or AVSG_E_RANGE. */
avsg_status avsg_fp8_quantize(const void *d_x, int32_t type, int32_t batch, int64_t rows, int64_t cols,
                              int64_t x_stride, int64_t x_batch_stride, const avsg_fp8 *out, void *stream);

/* The values that codes and scales stand for, as `type`, each product rounded once.
 * Limits as above. */
avsg_status avsg_fp8_dequantize(const avsg_fp8 *x, int32_t batch, int64_t rows, int64_t cols, void *d_out, int32_t type,
                                int64_t out_stride, int64_t out_batch_stride, void *stream);

/* out[i] = a[i] b[i]^T for i in [0, batch): a[i] is [m][k] with block_rows 1, b[i] is
 * [n][k] with block_rows 128, out[i] [m][n] of out_type with out_stride elements from row
 * to row and out_batch_stride from product to product.  k is a multiple of 16.
 * Products are those of the matrix instruction: exact, but those of eight neighbouring
 * columns are cut at 2^-13 of the largest one's power of two before they add up (in normal data
 * a result is off by some 2^-17 of the sum of its products' magnitudes); the eights' sums
 * add up in float32, and so do the blocks', times the product of both scales (which has to
 * be in float32's range).  A code of NaN makes
 * its results NaN.  m and n
 * are at most 4194240, k is below 2^30, out[i] has fewer than 2^24 tiles of 64 x 64 and
 * batch is at most 65535, or AVSG_E_RANGE. */
avsg_status avsg_fp8_matmul(const avsg_fp8 *a, const avsg_fp8 *b, int32_t batch, int64_t m, int64_t n, int64_t k,
                            void *d_out, int32_t out_type, int64_t out_stride, int64_t out_batch_stride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* AVSG_FP8_H */
