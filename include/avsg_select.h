/* avsg_select.h — C ABI of what makes a step's selection: the cache of 8-bit
 * index keys, and the scores over it with the positions that they select.
 *
 * A row of the key cache is one token position's index key, AVSG_KEY_ROW_BYTES
 * bytes: AVSG_KEY_DIM codes of 8 bits (two's complement, -127 to 127), then one
 * float32 scale; value = code * scale.  Rows of this size are the second kind that
 * avsg_step moves (row_bytes 132), which does not look into them.  The codes here are whole
 * numbers: rows with codes in 8-bit floating point have the same size, are not told
 * apart, and would be scored as whole numbers; only rows of avsg_key_append_rows, or of its
 * form, belong into a cache.  Queries are codes alike; what their scale multiplies
 * stands in their weights.
 *
 * A query token t has several index queries (heads) q[t][h] with weights w[t][h];
 * all meet the same keys.  The score of position p is
 *
 *   s[t][p] = float32( scale[p] * sum over h of w[t][h] * max(0, q[t][h] . key[p]) ),
 *
 * where the products of codes add up exactly in whole numbers and the sum over
 * the heads in 64 bits, always in the same order.  So a score does not depend on how the work is
 * split, and a selection is the same for one token as for a chunk of them.  A score is off the
 * exact one by its rounding to float32 and by at most 2^-47 of the sum of its terms'
 * magnitudes (35 roundings to 64 bits); positions that are closer than that may rank either way.
 *
 * Conventions are those of avsg_latent.h: the caller owns all memory, the calls are
 * asynchronous on the given stream, allocate nothing, never throw or abort, can
 * be captured into a HIP graph and keep no state, so calls on different streams are
 * independent as long as their outputs and workspaces are.
 * avsg_latent_last_error() describes the calling thread's last failure.
 */
#ifndef AVSG_SELECT_H
#define AVSG_SELECT_H

#include "avsg_latent.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AVSG_KEY_DIM 128
#define AVSG_KEY_ROW_BYTES 132
/* heads of a query token that avsg_select takes */
#define AVSG_SELECT_HEADS_MOST 128

/* Key rows of `batch` requests in pages, laid out like an avsg_cache: row x of
 * request r lies in page p = d_page_table[r * pages_per_request + x / page_rows]
 * (without a table p = r * pages_per_request + x / page_rows) at byte
 * p * page_stride + (x % page_rows) * row_stride of `base`.  Rows and pages
 * out of range are never written, and never read from. */
typedef struct avsg_key_cache {
    void *base;               /* device or pinned mapped host memory, 4-byte aligned */
    int64_t pages;            /* pages of the pool */
    int64_t page_stride;      /* bytes, a multiple of 4, at least page_rows * row_stride */
    int64_t row_stride;       /* bytes, a multiple of 4, at least AVSG_KEY_ROW_BYTES */
    int32_t batch;            /* requests */
    int32_t page_rows;        /* a power of two, or any count with pages_per_request 1 */
    int32_t pages_per_request;
    const int32_t *d_page_table; /* device [batch][pages_per_request], or NULL */
} avsg_key_cache;

/* New keys of a step or a prefill, and the index queries of the same tokens. */
typedef struct avsg_key_append {
    int64_t tokens;             /* T >= 0 */
    const void *d_key;          /* bfloat16 [T][128], not yet rotated; 16-byte aligned, like every row of it */
    int64_t key_stride;         /* elements from one token to the next, a multiple of 8 */
    const int32_t *d_request;   /* device [T]: the request of each token */
    const int64_t *d_position;  /* device [T]: its position, which is also its row */
    const float *d_angles;      /* device [positions][32][2]: cosine and sine of every pair; 16-byte aligned */
    int64_t positions;          /* rows of d_angles */
    int32_t rope_style;         /* AVSG_ROPE_* */
    int32_t rope_at;            /* first of the 64 columns that are rotated: 0 or 64; -1: none, and d_angles is not read */
    int32_t heads;              /* index queries per token, 0 = none */
    const void *d_q;            /* bfloat16 [T][heads][128], not yet rotated; 16-byte aligned rows */
    int64_t q_token_stride, q_head_stride;       /* elements, multiples of 8 */
    const float *d_weights;     /* [T][heads], or NULL: all 1 */
    int64_t weight_stride;      /* elements from one token to the next */
    void *d_q_out;              /* codes [T][heads][128]; 16-byte aligned rows */
    int64_t q_out_token_stride, q_out_head_stride; /* bytes, multiples of 16 */
    float *d_weights_out;       /* [T][heads]: weight times the query's scale */
    int64_t weight_out_stride;
} avsg_key_append;

/* Append: rotates 64 columns of each token's key by its position (pair (a, b) becomes
 * (a cos - b sin, a sin + b cos), in float32, every product and sum rounded),
 * quantises the 128 columns and writes the row: with a the largest magnitude,
 * code = x * (127 / a) rounded to the nearest, ties to even, scale = a / 127.
 * Below a = 2^-119 the codes and the scale are zero; a vector with an infinity or
 * a NaN has codes of zero and scale NaN (its score ranks with those not seen).
 * Queries are treated alike in the same launch.
 * A token whose request, position or page is out of range writes no row; one
 * whose position is negative, or not below `positions` where columns are rotated,
 * writes no row either and gets codes and weights of zero.  Two tokens of one call
 * with the same row race.  tokens * (1 + heads) is at most 2^28 - 16, or AVSG_E_RANGE. */
avsg_status avsg_key_append_rows(const avsg_key_cache *cache, const avsg_key_append *a, void *stream);

/* Read n rows back as bfloat16 [n][128] (16-byte aligned, out_stride elements from
 * row to row, a multiple of 8), code * scale rounded once.  Rows out of range read
 * as zeros.  n is at most 2^28 - 16, or AVSG_E_RANGE. */
avsg_status avsg_key_read_rows(const avsg_key_cache *cache, int64_t n, const int32_t *d_request,
                               const int64_t *d_position, void *d_out, int64_t out_stride, void *stream);

/* The selection of the step's query tokens. */
typedef struct avsg_selection {
    int32_t n_q;              /* query tokens per request, at least 1 */
    int32_t heads;            /* index queries per token, 1 to AVSG_SELECT_HEADS_MOST */
    int32_t longest;          /* positions [0, longest) are ranked; a multiple of block, at most the rows of a request */
    int32_t topk;             /* K positions are selected; a multiple of block, at most longest */
    int32_t block;            /* neighbouring positions that are selected together: a power of two, 1 to 128 */
    int32_t first;            /* positions [0, first) that a token sees are always taken, */
    int32_t recent;           /* and so are its last ones [len - recent, len) */
    const void *d_q;          /* codes [B][n_q][heads][128]; 16-byte aligned rows */
    int64_t q_token_stride, q_head_stride;   /* bytes, multiples of 16 */
    const float *d_weights;   /* [B][n_q][heads] */
    int64_t weight_stride;    /* elements from one token to the next */
    const int64_t *d_lens;    /* device [B][n_q]: positions a query token may see (no more than longest), or NULL: all of longest */
    int32_t *d_index;         /* device [B][n_q][K]: the positions selected, ascending (avsg_step's d_topk) */
    float *d_scores;          /* float32 [B][n_q][K / block]: the selected blocks' scores, or NULL */
} avsg_selection;

/* Bytes of device workspace avsg_select asks for (16-byte aligned; contents do not
 * matter before or after a call).  Scores of tokens are kept there between its
 * kernels; with less, down to avsg_select_workspace_least, it takes the tokens in
 * turns.  0 for sizes that avsg_select does not take. */
size_t avsg_select_workspace_bytes(int32_t batch, int32_t n_q, int32_t longest, int32_t block);
size_t avsg_select_workspace_least(int32_t longest, int32_t block);

/* Selects, for each query token, the K / block blocks of `block` positions with the
 * best scores, ties going to the lowest, and writes their positions in ascending
 * order.  A block's score is the largest of its positions'.  A position's is, by the first of
 * these that holds: minus infinity at or past the token's length (a negative length is 0);
 * infinity in [0, first) and [len - recent, len), whatever its row is; minus infinity where the
 * row does not exist or the score is NaN; the score.  So with fewer than K
 * positions to see, the selection goes on with the lowest others, and the K entries are
 * distinct positions below `longest` in any case: what avsg_step takes, and what
 * avsg_attend masks by their position.
 * Rows that no token of a request sees are not read; in place of a row that does not exist
 * the pool's first one is read, and counts for nothing.
 * batch * n_q is at most 2^19 and longest at most 2^30, or AVSG_E_RANGE. */
avsg_status avsg_select(const avsg_key_cache *cache, const avsg_selection *s, void *d_workspace,
                        size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* AVSG_SELECT_H */
