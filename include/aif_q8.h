/*
 * aif_q8.h -- C ABI of layers in 8 bits on MI355X (gfx950): rows that are summed,
 * normalised and left in 8-bit floating point, products of such rows with a
 * layer's weights, and the way in and out of the format.  They are the dense
 * layers of AIF's networks (arXiv 2511.12934: the heads of Sec. 1, the user
 * network of Sec. 3.1, the item network of Sec. 3.2) with a byte a value, twice
 * the matrix cores' rate of 16 bits and half the weights' bytes.
 *
 * Format.  A matrix of 8 bits holds a code in e4m3 (sign, 4 bits of exponent with
 * bias 7, 3 of mantissa, no infinity, 0x7f and 0xff no number) for each value and a
 * power of two for each block of 128 columns of a row (or of 128 rows by 128
 * columns: a layer's weights); the last block is smaller.  A block with largest
 * magnitude m is held with 2^e, e the smallest integer with m <= 448 * 2^e, kept
 * within -117..120, as a byte e + 127, and its values as the codes nearest to
 * value / 2^e, of two equally near the even one.  A block that holds a NaN or an
 * infinity has scale 1 and reads as NaN throughout.  Codes being floating point, a
 * power of two costs them no accuracy: off by 2^-4 of the value at most, from
 * 2^(e - 6) on, and by 2^(e - 10) below.  What a matrix holds stands exactly
 * in bf16 and in fp32 (beyond 2^128: as an infinity).
 * Scale bytes of a matrix that is read: 10..247, those that these calls write (others: the result is not defined).
 *
 * Conventions are those of aif.h: plain C, every call returns an aif_status and
 * enqueues nothing on failure (but where a HIP call fails, outputs hold anything),
 * DEVICE pointers belong to the device that was current at init, argument structs
 * are HOST memory read during the call, all device work is asynchronous on the caller's
 * stream.  The context holds nothing that a call changes but the text of its last
 * failure: calls on one context may run on any number of streams at once, one
 * thread at a time.  Each call is one launch and nothing else, and may be captured into a HIP graph.
 * The same call gives the same bits.  A call without rows is AIF_OK and does nothing.  Outputs must not overlap
 * each other or what the call reads, but where it says so below.  Nothing is written beside the rows and
 * columns named.
 */
#ifndef AIF_Q8_H
#define AIF_Q8_H

#include "aif.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct aif_q8_ctx aif_q8_ctx;

/* A matrix of 8 bits; its width, rows and block are the call's.  Widths are multiples of 8. */
typedef struct {
    void *codes;            /* DEVICE [rows, width] bytes, 16-byte aligned                                                    */
    void *scales;           /* DEVICE [rows or ceil(rows / 128), ceil(width / 128)] bytes, 4-byte aligned                     */
    int64_t stride;         /* bytes from one row of codes to the next: a multiple of 16 below 2^23 (0: width rounded up to one).
                               The bytes up to a multiple of 16 of a row that is read are read with the others and say nothing */
    int64_t scale_stride;   /* bytes from one row of scales to the next: a multiple of 4 (0: ceil(width / 128), rounded up to one).
                               The bytes up to a multiple of 4 are read with the others and say nothing                        */
} aif_q8_matrix;

/* Rows of dtype: DEVICE, 16-byte aligned, row i at i * stride elements, strides multiples of 16 bytes below 2^33 elements
 * (0: rows lie close).  Widths are multiples of 16 bytes (of 8 columns where 8 bits come out); of aif_q8_rows up to 16384. */
typedef struct {
    aif_dtype dtype;        /* of x, residual, weight, sum_out and out                                                        */
    int32_t n_rows;
    int32_t width;
    int32_t norm;           /* 0: y = h, and eps and weight say nothing; 1: the root mean square norm                         */
    float eps;              /* > 0 with norm                                                                                  */
    int32_t reserved;       /* 0                                                                                              */
    const void *x;          /* [n_rows, width]                                                                                */
    const void *residual;   /* [n_rows, width] or NULL                                                                        */
    const void *weight;     /* [width] or NULL: ones                                                                          */
    void *sum_out;          /* h, [n_rows, width] or NULL; may be x or residual itself (the same pointer and stride)          */
    void *out;              /* y, [n_rows, width] or NULL; may be x or residual too, if sum_out is not that one              */
    aif_q8_matrix q_out;    /* y in 8 bits, a block to 128 columns of a row; codes NULL: none                                 */
    int64_t x_stride;
    int64_t residual_stride;
    int64_t sum_stride;
    int64_t out_stride;
} aif_q8_rows_args;

typedef enum { AIF_Q8_NONE = 0, AIF_Q8_RELU = 1, AIF_Q8_GATE = 2 } aif_q8_activation;

typedef struct {
    aif_dtype dtype;        /* of bias, residual and out                                                                      */
    int32_t n_rows;         /* up to 2^30, and n_rows * n up to 2^44                                                          */
    int32_t k;              /* columns of a, w and up: up to 2^20, as n                                                       */
    int32_t n;              /* rows of w and up = columns of the result: a multiple of 16 bytes of dtype, of 8 for q_out      */
    int32_t activation;     /* aif_q8_activation                                                                              */
    int32_t reserved;       /* 0                                                                                              */
    aif_q8_matrix a;        /* [n_rows, k], a block to 128 columns of a row                                                   */
    aif_q8_matrix w;        /* [n, k], a block to 128 rows by 128 columns                                                     */
    aif_q8_matrix up;       /* as w, with AIF_Q8_GATE only (else codes NULL)                                                  */
    const void *bias;       /* DEVICE [n], 16-byte aligned, or NULL; not with AIF_Q8_GATE                                     */
    const void *residual;   /* rows of dtype [n_rows, n] or NULL                                                              */
    void *out;              /* rows of dtype [n_rows, n]; may be residual itself.  Either this ...                            */
    aif_q8_matrix q_out;    /* ... or [n_rows, n], a block to 128 columns of a row; the other NULL                            */
    int64_t residual_stride;
    int64_t out_stride;
} aif_q8_linear_args;

/* The way in and out.  block_rows: 1 (a block to 128 columns of a row) or 128 (a layer's weights). */
typedef struct {
    aif_dtype dtype;        /* of rows                                                                                        */
    int32_t n_rows;
    int32_t width;          /* a multiple of 8, up to 2^20                                                                    */
    int32_t block_rows;
    void *rows;             /* DEVICE [n_rows, width], as above; read by aif_q8_weights, written by aif_q8_values             */
    int64_t stride;
    aif_q8_matrix q;        /* written by aif_q8_weights, read by aif_q8_values                                               */
} aif_q8_convert_args;

/* A context on the current device.  *out is set only on AIF_OK. */
AIF_API aif_status aif_q8_init(aif_q8_ctx **out);

/* Frees the context; work enqueued through it goes on.  NULL is allowed. */
AIF_API void aif_q8_destroy(aif_q8_ctx *ctx);

/* Text of the last failure of this context (of the last failed aif_q8_init of the calling thread when ctx is NULL). */
AIF_API const char *aif_q8_last_error(const aif_q8_ctx *ctx);

/* h = x + residual,  y = h / sqrt(mean of h^2 over the row + eps) * weight,  in 64 bits, each output rounded once.
 * Errors: AIF_EINVAL (NULL, sizes, alignment, no output), AIF_ESHAPE (a width that is no multiple), AIF_ERANGE (a limit),
 * AIF_EDEVICE (a HIP call failed, or the current device is another one). */
AIF_API aif_status aif_q8_rows(aif_q8_ctx *ctx, const aif_q8_rows_args *args, void *hip_stream);

/* z_ij = sum_k a_ik w_jk + bias_j, then
 *   AIF_Q8_NONE z,  AIF_Q8_RELU max(z, 0) (NaN stays),  AIF_Q8_GATE z / (1 + exp(-z)) * sum_k a_ik up_jk,
 * then + residual_ij; sums in fp32 (terms below 2^-126 may count as nothing), rounded once.  With AIF_F32 every product enters them whole.  With
 * AIF_BF16 the matrix cores add the products of eight neighbouring columns (8 c .. 8 c + 7) at a time and cut off what lies 13
 * binary places below the exponent of their largest, and the sums are fp32 from there on: 1.5 - 2.3 10^-5 of results in 2-norm, at twice the rate.
 * The gate's z / (1 + exp(-z)) is off by (|z| / 2 + 6.8) 2^-23 of itself and 2^-150 |z| at most, and may count as nothing below 2^-126, from z = -92 on.
 * How the sum over k is shared out, and with it the order of the additions, depends on the sizes of the call.  Errors as aif_q8_rows. */
AIF_API aif_status aif_q8_linear(aif_q8_ctx *ctx, const aif_q8_linear_args *args, void *hip_stream);

/* Rows (or a layer's weights) of dtype into 8 bits.  Errors as aif_q8_rows. */
AIF_API aif_status aif_q8_weights(aif_q8_ctx *ctx, const aif_q8_convert_args *args, void *hip_stream);

/* The values that codes and scales stand for, rounded to dtype (which they are in but for infinities).  Errors as aif_q8_rows. */
AIF_API aif_status aif_q8_values(aif_q8_ctx *ctx, const aif_q8_convert_args *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* AIF_Q8_H */
