/* avsg_latent.h — C ABI of the operators around the sparse gather: the cache of
 * latent key/value rows that a step's gather reads from (avsg.h), the
 * attention over the rows that it placed, and the 4-bit microscaled
 * quantisation and product that serve the projections before and after it.
 *
 * A cache row is one token position.  It holds a latent vector of
 * AVSG_LATENT_DIM values, which is the position's key and its value for every
 * head, and AVSG_ROPE_DIM values of the key that carry the position:
 *   AVSG_ROWS_BF16  1152 bytes: 512 latent values, then 64 rotated ones, bfloat16
 *                   (the row of Appendix D: (512 + 64) * 2 bytes);
 *   AVSG_ROWS_MX4   400 bytes: 256 bytes of 4-bit codes of the latent values
 *                   (column 2i in the low half of byte i), 16 bytes of scales,
 *                   one per AVSG_MX4_BLOCK columns, then the 64 rotated values in
 *                   bfloat16.  A row fetched over the host link costs 0.35 of a
 *                   bfloat16 row's bytes.
 * Either is a row_bytes[0] of avsg_config, so avsg_step moves such rows as they are.
 *
 * Microscaled 4-bit values ("mx4"): blocks of 32 consecutive columns share one
 * scale byte s; code c stands for v(c) * 2^(s - 127) with
 * v = 0, 0.5, 1, 1.5, 2, 3, 4, 6 for c = 0..7 and their negatives for c = 8..15.
 * s = 255 makes all 32 values NaN.
 *
 * Conventions are those of avsg.h: the caller owns all memory, the calls are
 * asynchronous on the given stream and never throw, abort or allocate, and can
 * be captured into a HIP graph (they enqueue kernels only).  They keep no state,
 * so calls on different streams are independent as long as their outputs and
 * workspaces are.  avsg_latent_last_error() describes the calling thread's last
 * failure.
 */
#ifndef AVSG_LATENT_H
#define AVSG_LATENT_H

#include "avsg.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AVSG_LATENT_DIM 512
#define AVSG_ROPE_DIM 64
#define AVSG_MX4_BLOCK 32

/* Row formats. */
#define AVSG_ROWS_BF16 0
#define AVSG_ROWS_MX4 1

/* Which columns of a rotated part form a pair. */
#define AVSG_ROPE_PAIRS 0   /* 2i and 2i + 1 */
#define AVSG_ROPE_HALVES 1  /* i and i + 32 */

/* Element types of plain matrices. */
#define AVSG_BF16 0
#define AVSG_F32 1

/* Bytes of a row of a format (1152 or 400), 0 for an unknown format. */
size_t avsg_row_bytes(int32_t format);

/* Cache rows of `batch` requests in pages.  Row x of request r lies in page
 * p = d_page_table[r * pages_per_request + x / page_rows] of the pool, at byte
 * p * page_stride + (x % page_rows) * row_stride of `base`; without a table
 * p = r * pages_per_request + x / page_rows.  Rows outside
 * [0, pages_per_request * page_rows) and pages outside [0, pages) are never
 * touched.
 * `base` is device memory, or pinned mapped host memory (avsg_host_alloc).  The
 * slot buffers of avsg_step are such a cache of one page of S rows per request;
 * so are the host rows of avsg_create, when they lie at equal distances. */
typedef struct avsg_cache {
    void *base;               /* 16-byte aligned */
    int64_t pages;            /* pages of the pool */
    int64_t page_stride;      /* bytes, a multiple of 16, at least page_rows * row_stride */
    int64_t row_stride;       /* bytes, a multiple of 16, at least avsg_row_bytes(format) */
    int32_t format;           /* AVSG_ROWS_* */
    int32_t batch;            /* requests */
    int32_t page_rows;        /* a power of two, or any count with pages_per_request 1 */
    int32_t pages_per_request;
    const int32_t *d_page_table; /* device [batch][pages_per_request], or NULL */
} avsg_cache;

/* New rows of a step or a prefill. */
typedef struct avsg_append {
    int64_t tokens;             /* T >= 0 */
    const void *d_latent;       /* bfloat16 [T][512]; 16-byte aligned, like every row of it */
    int64_t latent_stride;      /* elements from one token to the next, a multiple of 8 */
    const void *d_rope;         /* bfloat16 [T][64], not yet rotated; likewise */
    int64_t rope_stride;
    const int32_t *d_request;   /* device [T]: the request of each token */
    const int64_t *d_position;  /* device [T]: its position, which is also its row */
    const float *d_angles;      /* device [positions][32][2]: cosine and sine of every pair; 16-byte aligned */
    int64_t positions;          /* rows of d_angles */
    int32_t rope_style;         /* AVSG_ROPE_* */
    int32_t heads;              /* heads of the queries rotated along with the keys, 0 = none */
    const void *d_q;            /* bfloat16 [T][heads][64], not yet rotated; 16-byte aligned rows */
    int64_t q_token_stride, q_head_stride;       /* elements, multiples of 8 */
    void *d_q_out;              /* bfloat16 [T][heads][64]: the rotated queries; 16-byte aligned rows */
    int64_t q_out_token_stride, q_out_head_stride;
} avsg_append;

/* Append: rotates each token's 64 positional values by its position (pair (a,
 * b) becomes (a cos - b sin, a sin + b cos), in float32, rounded once to
 * bfloat16), brings the latent values into the cache's format and writes the
 * row.  The queries of the same tokens are rotated in the same launch.
 * A token whose request, position or page is out of range writes no row; one
 * whose position lies outside [0, positions) writes no row either and gets
 * queries of zeros (padding tokens have position -1).  d_q_out may be d_q.  Two
 * tokens of one call with the same row race.  tokens * (1 + heads / 8, rounded up) is
 * at most 67108860, what a launch takes, or AVSG_E_RANGE. */
avsg_status avsg_kv_append(const avsg_cache *cache, const avsg_append *a, void *stream);

/* Read n rows back as bfloat16 [n][576] (latent, then rotated part; 16-byte
 * aligned, out_stride elements from row to row, a multiple of 8).  Rows out of
 * range read as zeros.  n is at most 67108860, or AVSG_E_RANGE. */
avsg_status avsg_kv_read(const avsg_cache *cache, int64_t n, const int32_t *d_request,
                         const int64_t *d_position, void *d_out, int64_t out_stride, void *stream);

/* Attention of the step's query tokens over cache rows. */
typedef struct avsg_attention {
    int32_t n_q;              /* query tokens per request */
    int32_t heads;            /* H query heads; all read the same rows */
    int32_t topk;             /* K entries per query token */
    float scale;              /* of the scores */
    const void *d_q;          /* bfloat16 [B][n_q][H][576]: 512 values against the latent part, 64 against the rotated one */
    int64_t q_token_stride, q_head_stride;   /* elements, multiples of 8; 16-byte aligned rows */
    const int32_t *d_rows;    /* device [B][n_q][K]: the row of each entry (avsg_step's d_slots), or NULL: entry i is row i */
    const int32_t *d_index;   /* device [B][n_q][K]: the position of each entry (avsg_step's d_topk), or NULL: entry i has position i */
    const int64_t *d_lens;    /* device [B][n_q]: positions a query token may see, or NULL: all */
    void *d_out;              /* bfloat16 [B][n_q][H][512] */
    int64_t out_token_stride, out_head_stride; /* elements, multiples of 8; 16-byte aligned rows */
    float *d_lse;             /* float32 [B][n_q][H]: log of the sum of exp(score), or NULL */
} avsg_attention;

/* Bytes of device workspace avsg_attend needs (256-byte aligned; contents do
 * not matter before or after a call), 0 when it needs none.  They are those of a call
 * of exactly these sizes: one of fewer requests, tokens, heads or entries, which more
 * workgroups share, may need more.  AVSG_ATTEND_WORKSPACE_MOST are enough for any call. */
#define AVSG_ATTEND_WORKSPACE_MOST 33685504
size_t avsg_attend_workspace_bytes(int32_t batch, int32_t n_q, int32_t heads, int32_t topk);

/* out = sum_i softmax_i(scale * q . key_i) * value_i over the entries i of a
 * query token that count: their position lies in [0, len) and their row exists.
 * Rows of entries that do not count are not read.  A token without any gets
 * zeros, and minus infinity in d_lse.  Products take bfloat16 operands (4-bit
 * rows are expanded exactly; a probability is a sum of two operands and keeps 12
 * bits at least, or is off by 2^-19 of its token's largest) and add up in float32,
 * as do maxima and sums.  No sum exceeds the rows' largest value, so what is finite
 * in the rows is finite in the result.  batch * n_q is at most 2^19, heads at most
 * 4096, and batch * n_q * heads at most what one launch takes (2^26 always), or AVSG_E_RANGE. */
avsg_status avsg_attend(const avsg_cache *cache, const avsg_attention *a, void *d_workspace,
                        size_t workspace_bytes, void *stream);

/* mx4 form of x (AVSG_BF16 or AVSG_F32, [rows][cols], cols a multiple of 32;
 * rows 16-byte aligned, x_stride elements apart): d_codes [rows][cols / 2] and
 * d_scales [rows][cols / 32], contiguous.  A block's scale is the power of two
 * that brings its largest magnitude into [3.5, 7), values are rounded to the
 * nearest code, ties to the even code; scales are at least 2^-125, and at most
 * 2^125 (magnitudes above 7 * 2^125 become 6 * 2^125).  A block that holds an
 * infinity or a NaN gets scale 255.  rows * cols is at most 2^35 - 2048 here
 * and in avsg_mx4_dequantize, or AVSG_E_RANGE. */
avsg_status avsg_mx4_quantize(const void *d_x, int32_t type, int64_t rows, int64_t cols, int64_t x_stride,
                              void *d_codes, void *d_scales, void *stream);

/* A matrix, or a batch of them, in mx4 form.  Codes are 16-byte aligned and their
 * strides multiples of 16 bytes where k > 32 columns are read by a product. */
typedef struct avsg_mx4 {
    const void *d_codes;
    const void *d_scales;
    int64_t code_stride, code_batch_stride;    /* bytes from row to row, from matrix to matrix */
    int64_t scale_stride, scale_batch_stride;
} avsg_mx4;

/* The values that [rows][cols] codes stand for, as `type`; exact for scales from 2^-125 to 2^125. */
avsg_status avsg_mx4_dequantize(const avsg_mx4 *x, int64_t rows, int64_t cols, void *d_out, int32_t type,
                                int64_t out_stride, void *stream);

/* out[i] = a[i] b[i]^T for i in [0, batch): a[i] is [m][k], b[i] is [n][k], both
 * mx4, out[i] [m][n] of out_type with out_stride elements from row to row and
 * out_batch_stride from product to product.  k is a multiple of 32.  Products
 * are exact and add up in float32.  m, n and k are below 2^30, out[i] has fewer than 2^24
 * tiles of 128 x 128 and batch is at most 65535, or AVSG_E_RANGE. */
avsg_status avsg_mx4_matmul(const avsg_mx4 *a, const avsg_mx4 *b, int32_t batch, int64_t m, int64_t n,
                            int64_t k, void *d_out, int32_t out_type, int64_t out_stride,
                            int64_t out_batch_stride, void *stream);

/* What the calling thread's last failed call of this header did not like. */
const char *avsg_latent_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* AVSG_LATENT_H */
