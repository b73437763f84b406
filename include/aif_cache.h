/*
 * aif_cache.h -- C ABI of the user cache on MI355X (gfx950): behaviour
 * sequences that the asynchronous phase of AIF (arXiv 2511.12934, Sec. 3.1)
 * leaves for the real-time phase, held in pages of 4 bits, and what reads,
 * extends, branches and moves them.
 *
 * A sequence is a user's keys and values, one row of n_kv_heads * d_head
 * features each per behaviour (for instance U^_seq of aif_user.h, which is
 * both).  Rows enter by aif_cache_append, one new behaviour or a whole history
 * at a time, and are read in place by aif_cache_attend -- the operator of Eq. 3
 * with candidates (or the one next behaviour) as queries -- or unpacked by
 * aif_cache_read into the dense tensors that aif_score_batch takes.
 *
 * Format.  A head's d_head features are cut into blocks of 32, the last one
 * shorter.  A block with largest magnitude m is held with the power of two
 * 2^e, e the smallest integer with m <= 6 * 2^e, kept within -125..125, as a
 * byte e + 127, and its features as signed codes of the magnitudes
 * {0, 1/2, 1, 3/2, 2, 3, 4, 6} * 2^e, each the nearest one (a tie goes to the
 * one at an even place of that list, what is beyond the largest to it): off by
 * at most 2^e, a third of m, from 4 * 2^e on, half of that from 2 * 2^e on and a quarter below.
 * A block that holds a NaN or an infinity reads as NaN throughout.
 * What the cache holds stands exactly in bf16 and in fp32.
 *
 * Pages.  The caller provides the pool: n_pages pages of
 * aif_cache_page_bytes() bytes (4.25 bits a feature, d_head rounded up to a
 * multiple of 32).  A page holds page_len consecutive rows of one sequence,
 * all heads.  Sequences are known by numbers 0 .. max_seqs - 1 and empty at
 * first; the context keeps which pages belong to which, lowest free page
 * first.  A fork shares pages: a shared page is written by nobody, and a
 * sequence that appends into its shared last page gets a copy of it first.
 *
 * Conventions are those of aif.h: plain C, every call returns an aif_status,
 * changes and enqueues nothing on failure (but see AIF_EDEVICE below), DEVICE
 * pointers belong to the device that was current at init, HOST arrays are read
 * during the call, all device work is asynchronous on the caller's stream, the
 * library owns its context and workspace and borrows the pool for the life of
 * the context and the request tensors until the enqueued work has completed.
 * The book-keeping (lengths, pages in use) is the host's and takes effect at
 * once; the pages' contents follow in the order of the stream, so calls on one
 * context belong on one stream, or on streams that the caller orders.  A
 * context serves one thread at a time.  Not capturable into a HIP graph: under
 * capture the calls that enqueue return AIF_EINVAL.
 * AIF_EDEVICE: a HIP call failed, or the current device is another one.  In the
 * second case nothing has changed.  In the first, outputs of attend and read
 * hold anything, and what the device holds of the sequences that append and trim
 * name, fork and copy make, or compact moves (any) is not known: these are empty
 * afterwards.  The other sequences are as they were.
 */
#ifndef AIF_CACHE_H
#define AIF_CACHE_H

#include <stddef.h>

#include "aif.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct aif_cache_ctx aif_cache_ctx;

typedef struct {
    aif_dtype dtype;        /* type of appended and read rows, queries and outputs                   */
    int32_t n_heads;        /* query heads, a multiple of n_kv_heads; head h reads kv head h / (n_heads / n_kv_heads) */
    int32_t n_kv_heads;     /* heads of a key or value row                                           */
    int32_t d_head;         /* a multiple of 16 bytes in dtype, up to 256                            */
    float scale;            /* of the scores, > 0, up to 2.35e38; 0 stands for 1 / sqrt(d_head)      */
    int32_t page_len;       /* rows of a page: a multiple of 32, 32..1024; a page has up to 2^29 bytes */
    int32_t n_pages;        /* pages of the pool                                                     */
    int32_t max_seqs;       /* sequence numbers are 0 .. max_seqs - 1                                */
    int32_t max_len;        /* longest sequence, in rows: up to 2^30, and 2^23 pages                 */
    int32_t max_requests;   /* entries of one call                                                   */
    int32_t max_queries;    /* largest n_q of one entry of aif_cache_attend                          */
} aif_cache_config;

/* Rows for the end of a sequence.  keys and vals: DEVICE, 16-byte aligned, row i at i * stride elements, strides multiples
 * of 16 bytes below 2^33 elements (0: rows lie close, stride = n_kv_heads * d_head); vals may alias keys. */
typedef struct {
    int32_t seq;
    int32_t n_rows;         /* >= 0 */
    const void *keys;       /* [n_rows, n_kv_heads * d_head] */
    const void *vals;
    int64_t key_stride;
    int64_t val_stride;
} aif_cache_append_req;

/* Queries over a sequence.  Query i of any head sees row j where j < len, j <= p_i, and window = 0 or j > p_i - window or
 * j < sinks; p_i = positions[i], or len - 1 without positions.  Rows that aif_cache_trim dropped are seen by nobody.
 * q and out: DEVICE, 16-byte aligned, strides as above (0: n_heads * d_head). */
typedef struct {
    int32_t seq;
    int32_t n_q;            /* 0..max_queries */
    const void *q;          /* [n_q, n_heads, d_head] */
    void *out;              /* [n_q, n_heads, d_head] */
    float *lse_out;         /* DEVICE [n_q, n_heads] or NULL: log of the sum of exp(score) over the rows seen */
    const int32_t *positions; /* DEVICE [n_q] or NULL; any value: below 0 sees nothing */
    int64_t q_stride;
    int64_t out_stride;
    int32_t sinks;          /* >= 0; without a window it says nothing */
    int32_t window;         /* >= 0; 0 = no window */
} aif_cache_attend_req;

/* Rows [first, first + n_rows) of a sequence as the values they stand for.  Strides as above; either output may be NULL. */
typedef struct {
    int32_t seq;
    int32_t first;
    int32_t n_rows;
    int32_t reserved;       /* 0 */
    void *keys_out;         /* DEVICE [n_rows, n_kv_heads * d_head] */
    void *vals_out;
    int64_t key_stride;
    int64_t val_stride;
} aif_cache_read_req;

/* Bytes of a page of such a cache (dtype, n_kv_heads, d_head and page_len are read); 0 where a context could not be made. */
AIF_API size_t aif_cache_page_bytes(const aif_cache_config *config);

/* A context over a pool of n_pages pages (DEVICE, 64-byte aligned, writable, borrowed until aif_cache_destroy or
 * aif_cache_swap_pool; its contents need not be set).  Synchronous.  *out is set only on AIF_OK. */
AIF_API aif_status aif_cache_init(const aif_cache_config *config, void *pool, aif_cache_ctx **out);

/* Frees the context and its workspace; the caller has synchronised its streams.  NULL is allowed. */
AIF_API void aif_cache_destroy(aif_cache_ctx *ctx);

/* Text of the last failure of this context (of the last failed aif_cache_init of the calling thread when ctx is NULL). */
AIF_API const char *aif_cache_last_error(const aif_cache_ctx *ctx);

/* Rows to the ends of n sequences, each named once.  Errors: AIF_EINVAL (NULL, negative or misaligned sizes, a sequence
 * named twice), AIF_ERANGE (a number outside the context, more than max_len rows, not enough free pages). */
AIF_API aif_status aif_cache_append(aif_cache_ctx *ctx, const aif_cache_append_req *reqs, int32_t n, void *hip_stream);

/* Softmax attention of n entries' queries over their sequences; a sequence may be named any number of times.
 *   out_i = sum_j w_ij v_j,  w_i = softmax over the rows j that query i sees of scale * <q_i, k_j>
 * A query that sees no row, or whose scores are all minus infinity, gives zeros and lse = -inf.  Sums and weights are fp32;
 * in bf16 the weights are rounded to bf16 where they meet the values.  What a query does not see does not reach it,
 * NaN included.  How a long sequence is shared out, and with it the order of the additions, depends on the call; the same call
 * gives the same bits.  The outputs must not overlap the pool, the queries or each other.
 * Errors: AIF_EINVAL, AIF_ERANGE (a number outside the context; more than 2^31 - 1 queries times heads of a kv head in the
 * call, or more than about 10^9 of them in large entries). */
AIF_API aif_status aif_cache_attend(aif_cache_ctx *ctx, const aif_cache_attend_req *reqs, int32_t n, void *hip_stream);

/* Unpacks rows.  Errors: AIF_EINVAL; AIF_ERANGE (rows at or beyond the sequence's length, or dropped by aif_cache_trim;
 * more than about 10^9 rows in a call). */
AIF_API aif_status aif_cache_read(aif_cache_ctx *ctx, const aif_cache_read_req *reqs, int32_t n, void *hip_stream);

/* src, dst: HOST arrays of n sequence numbers.  dst[i], which must be empty and named once, becomes what src[i] is, sharing
 * its pages.  Errors: AIF_EINVAL (dst[i] not empty or named twice, also as a source), AIF_ERANGE (a number outside the context). */
AIF_API aif_status aif_cache_fork(aif_cache_ctx *ctx, const int32_t *src, const int32_t *dst, int32_t n, void *hip_stream);

/* The same with pages of its own for dst[i].  Also AIF_ERANGE where there are not enough free pages. */
AIF_API aif_status aif_cache_copy(aif_cache_ctx *ctx, const int32_t *src, const int32_t *dst, int32_t n, void *hip_stream);

/* Sequences become empty; pages that no other one shares are free.  Host-side only: work enqueued earlier still reads them,
 * later calls on the stream may write them.  A number may be named twice.  Errors: AIF_EINVAL, AIF_ERANGE. */
AIF_API aif_status aif_cache_free(aif_cache_ctx *ctx, const int32_t *seqs, int32_t n);

/* The last rows of a sequence go: its length becomes len, pages beyond it are given back.  Host-side only, like
 * aif_cache_free.  Errors: AIF_EINVAL, AIF_ERANGE (len < 0 or beyond the length, or inside a page that was dropped). */
AIF_API aif_status aif_cache_truncate(aif_cache_ctx *ctx, int32_t seq, int32_t len);

/* Pages of n sequences that lie wholly behind the first sinks rows and before the last window rows are dropped and given back:
 * no query at len - 1 or later with that window and no more sinks would see them.  The rows that stay keep their numbers and the sequence its length.
 * window >= 1.  A number may be named twice.  Errors: AIF_EINVAL, AIF_ERANGE. */
AIF_API aif_status aif_cache_trim(aif_cache_ctx *ctx, const int32_t *seqs, int32_t n, int32_t sinks, int32_t window, void *hip_stream);

/* Moves pages until those in use are the first ones of the pool, whoever shares them; *n_used (HOST, may be NULL) becomes
 * their number. */
AIF_API aif_status aif_cache_compact(aif_cache_ctx *ctx, int32_t *n_used, void *hip_stream);

/* Later calls use another pool of n_pages pages that holds what the first pages of this one did: the caller has copied the
 * pages in use, after aif_cache_compact.  Host-side only; the old pool is the caller's again once enqueued work has
 * completed.  Errors: AIF_EINVAL (NULL, misaligned, n_pages < 1), AIF_ERANGE (a page in use at or beyond n_pages), AIF_ENOMEM. */
AIF_API aif_status aif_cache_swap_pool(aif_cache_ctx *ctx, void *pool, int32_t n_pages);

/* Length of a sequence; -1 for a number outside the context or a NULL context. */
AIF_API int32_t aif_cache_len(const aif_cache_ctx *ctx, int32_t seq);

/* Pages that no sequence uses; -1 for NULL. */
AIF_API int32_t aif_cache_free_pages(const aif_cache_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* AIF_CACHE_H */
