/*
 * hpacmlt.h -- what a surrogate's training step needs besides its layers in
 * 8-bit integers, a companion of hpacml.h and hpacml8.h: dense layers in 8-bit
 * floating point with a scale for each block of 128 values, their backward
 * pass, group norm with an activation on channels-last records, and the norm
 * and clipping of gradients.
 *
 * Conventions are those of hpacml8.h: device pointers on the current HIP
 * device, a hipStream_t passed as void*, statuses instead of exceptions, every
 * check done on the host before anything is enqueued.  A matrix is row-major
 * with a row pitch in elements; a row is a point of the sweep.  The library
 * verifies that every operand is device memory of the current device and lies
 * inside its allocation (HPACML_E_INVAL, HPACML_E_RANGE), and that nothing
 * written overlaps another operand (HPACML_E_ALIAS; rows of one record with
 * equal pitches may interleave).  Calls allocate nothing; what they need beyond
 * their operands is scratch memory of the caller (16-byte aligned), whose
 * contents mean nothing between calls.  No call synchronises, except the
 * creation and destruction of a set of gradients; none uses atomic operations:
 * equal calls give equal bits.  Calls with operands and scratch of their own
 * may overlap on different streams.
 */
#ifndef HPACMLT_H
#define HPACMLT_H

#include "hpacml.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- matrices in 8-bit floating point --------------------------------------
 * A value is e4m3: a sign, four bits of exponent, three of fraction; the
 * largest is 448, steps below 2^-6 are 2^-9.  A block of values shares a scale
 * 2^e, the smallest with max |v| <= 448 * 2^e (e at least -126), and has the
 * codes v / 2^e, rounded to e4m3, ties to even.  A code times its scale is
 * exact in bf16 and in fp32 (below 2^-126 it may count as 0).  A block with an
 * infinity, a NaN or a magnitude of 0x1.Fp127 and more, which would round to
 * 2^128, makes NaN of every result that it reaches.
 *
 * A matrix is rows by width, its blocks 128 values of a row (the last one may
 * be shorter), and a product takes two such matrices along their width.  The
 * order of codes and scales in memory is the library's own: the buffers are
 * written by hpacmlt_quantize and read by the calls below. */
#define HPACMLT_BLOCK 128

typedef struct {
    void *codes;          /* DEVICE, 16-byte aligned, of hpacmlt_matrix_bytes */
    void *scales;         /* DEVICE, 16-byte aligned, of hpacmlt_matrix_bytes */
    int64_t rows, width;  /* rows >= 0, width >= 0; each up to INT32_MAX, fewer than 2^24 blocks of 128 x 128 */
} hpacmlt_matrix;

/* Bytes of a matrix's buffers. */
hpacml_status hpacmlt_matrix_bytes(int64_t rows, int64_t width, size_t *codes, size_t *scales);

/* Codes and scales of x [rows][width], type HPACML_F32 or HPACML_BF16.
 *   by_row (may be NULL): the matrix x, its blocks 128 columns of a row.
 *   by_column (may be NULL, but not both): the matrix x^T (width rows of
 *   `rows` values), its blocks 128 rows of a column.
 *   square: nonzero makes blocks of 128 x 128 values of x instead, so that
 *   by_row and by_column hold the same codes (weights).
 * Asynchronous on `stream`. */
hpacml_status hpacmlt_quantize(const void *x, int32_t dtype, int64_t ldx, int64_t rows, int64_t width,
                               const hpacmlt_matrix *by_row, const hpacmlt_matrix *by_column, int32_t square,
                               void *stream);

/* What `m` stands for, as x [rows][width] of type HPACML_F32 or HPACML_BF16.
 * Asynchronous on `stream`. */
hpacml_status hpacmlt_load(const hpacmlt_matrix *m, void *x, int32_t dtype, int64_t ldx, void *stream);

/* y [p->rows][q->rows] (+)= act(p q^T + b): y_ij = act(sum_k p_ik q_jk + b_j),
 * products exact, sums in fp32, rounded once to y's type.  (Where y is bf16 the
 * 8-bit matrix instruction may drop of each product what is below 2^-13 of the
 * largest of its eight neighbours: less than 2^-10 of the sum of magnitudes, for
 * values without a common sign about 2^-16 of the result.  Where y is fp32 nothing
 * is dropped.)
 *   y_dtype: HPACML_F32 or HPACML_BF16; b: fp32 [q->rows] or NULL;
 *   act: HPACML_ACT_* (a ReLU keeps a NaN);
 *   accumulate: nonzero adds to y, which is fp32 then, without b and act.
 * Width zero: the sum is 0.  Asynchronous on `stream`. */
hpacml_status hpacmlt_product(const hpacmlt_matrix *p, const hpacmlt_matrix *q, const float *b, int32_t act,
                              void *y, int32_t y_dtype, int64_t ldy, int32_t accumulate, void *scratch,
                              size_t scratch_bytes, void *stream);
/* Bytes of scratch hpacmlt_product needs for these sizes. */
hpacml_status hpacmlt_product_scratch(int64_t p_rows, int64_t q_rows, int64_t width, size_t *bytes);

/* ---- a dense layer ------------------------------------------------------------
 * y [rows][W->rows] = act(x W^T + b) for x [rows][W->width]: x is quantized by
 * row, then as hpacmlt_product.  `W` is quantized by row with `square` blocks
 * where hpacmlt_backward is to be the gradient of the same layer.
 *   x_dtype, y_dtype: HPACML_F32 or HPACML_BF16; b: fp32 [W->rows] or NULL;
 *   keep (may be NULL): x by column (W->width rows of `rows`), for
 *   hpacmlt_backward. */
hpacml_status hpacmlt_linear_run(const hpacmlt_matrix *W, const float *b, const void *x, int32_t x_dtype,
                                 int64_t ldx, int64_t rows, void *y, int32_t y_dtype, int64_t ldy, int32_t act,
                                 const hpacmlt_matrix *keep, void *scratch, size_t scratch_bytes, void *stream);
/* Bytes of scratch hpacmlt_linear_run needs (with or without `keep`). */
hpacml_status hpacmlt_linear_scratch(const hpacmlt_matrix *W, int64_t rows, size_t *bytes);

/* The layer's backward pass from its input kept by column and the gradient dy
 * [rows][n_out] of its outputs (rows = kept->width, n_in = kept->rows):
 *     dz = dy, 0 where y <= 0 (y NULL: dz = dy)
 *     dw[j][k] (+)= sum_i dz_ij x_ik, dz quantized by column
 *     dx[i][k]  =   sum_j dz_ij W_jk, dz quantized by row
 *     db[j]    (+)= sum_i dz_ij, of dz itself
 *   dtype: HPACML_F32 or HPACML_BF16, the type of dy, y [rows][n_out] (the
 *   layer's outputs behind a ReLU, or NULL) and dx [rows][n_in]; dw
 *   [n_out][n_in] and db [n_out] are fp32;
 *   Wt: the weights by column (n_in rows of n_out), for dx.
 * Any of dw, db, dx may be NULL (not wanted); kept->codes and kept->scales are
 * read for dw only.  accumulate: nonzero adds to dw and db, zero sets them.
 * Zero rows: dw and db are set to 0 (accumulate: left). */
hpacml_status hpacmlt_backward(const hpacmlt_matrix *kept, const void *dy, const void *y, int32_t dtype,
                               int64_t lddy, int64_t ldy, int32_t n_out, const hpacmlt_matrix *Wt, float *dw,
                               int64_t lddw, float *db, void *dx, int64_t lddx, int32_t accumulate, void *scratch,
                               size_t scratch_bytes, void *stream);
/* Bytes of scratch hpacmlt_backward needs; want_*: which outputs are wanted. */
hpacml_status hpacmlt_backward_scratch(int64_t rows, int64_t n_in, int32_t n_out, int32_t want_dw, int32_t want_db,
                                       int32_t want_dx, size_t *bytes);

/* ---- group norm with an activation, channels last -------------------------------
 * x [images * points][channels]; a group is channels / groups neighbouring
 * channels.  Over an image's points and a group's channels together (n values)
 *     mean = sum x / n    rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)
 *     z = (x - mean) * (rstd * gamma) + beta     y = act(z)
 * Sums are in 64 bits, mean and rstd are rounded to fp32, what follows is in
 * fp32 (which x - mean has to fit), y rounded once to its type, which is x's.
 *   dtype: HPACML_F32 or HPACML_BF16; gamma, beta: fp32 [channels] or NULL (1
 *   and 0); eps >= 2^-126, finite; act: HPACML_ACT_* or HPACMLT_ACT_SILU (z / (1 +
 *   exp(-z))); mean, rstd: fp32 [images][groups], for the backward pass, or
 *   both NULL.  channels: 1..HPACMLT_MAX_CHANNELS, a multiple of groups.
 * An image with an infinity or a NaN in a group has NaNs there.  points is at
 * least 1; images may be 0. */
#define HPACMLT_ACT_SILU 2
#define HPACMLT_MAX_CHANNELS 16384

hpacml_status hpacmlt_group_norm(const void *x, int32_t dtype, int64_t ldx, int64_t images, int64_t points,
                                 int32_t channels, int32_t groups, const float *gamma, const float *beta, float eps,
                                 int32_t act, void *y, int64_t ldy, float *mean, float *rstd, void *scratch,
                                 size_t scratch_bytes, void *stream);

/* Its backward pass from the gradient dy of y: g = dy act'(z) and
 *     dgamma_c (+)= sum g (x - mean) rstd     dbeta_c (+)= sum g
 *     dx = rstd (g gamma - m1 - (x - mean) rstd m2)
 * with m1 and m2 the means of g gamma and g gamma (x - mean) rstd over image
 * and group, in fp32, whose range sums of g (x - mean) have to keep.  A ReLU's
 * act' is 0 where z <= 0 and 1 elsewhere.
 *   dy, dx: x's type; dx, dgamma, dbeta may be NULL (not wanted); gamma, beta,
 *   act as given to hpacmlt_group_norm, mean and rstd as it wrote them.
 * accumulate: nonzero adds to dgamma and dbeta, zero sets them (no images: to
 * 0). */
hpacml_status hpacmlt_group_norm_backward(const void *x, int32_t dtype, int64_t ldx, int64_t images, int64_t points,
                                          int32_t channels, int32_t groups, const float *gamma, const float *beta,
                                          int32_t act, const float *mean, const float *rstd, const void *dy,
                                          int64_t lddy, void *dx, int64_t lddx, float *dgamma, float *dbeta,
                                          int32_t accumulate, void *scratch, size_t scratch_bytes, void *stream);
/* Bytes of scratch of hpacmlt_group_norm (backward 0) and
 * hpacmlt_group_norm_backward (backward 1). */
hpacml_status hpacmlt_group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels,
                                         int32_t groups, int32_t backward, size_t *bytes);

/* ---- the norm of many gradients, and clipping ------------------------------------ */
typedef struct {
    const void *from;        /* DEVICE: the gradient, `count` values one after another */
    void *to;                /* where clipping writes it; `from` itself: in place */
    int64_t count;           /* >= 0; of no values: the pointers are not looked at */
    int32_t from_dtype;      /* HPACML_F32 or HPACML_BF16 */
    int32_t to_dtype;        /* the same; in place: from_dtype */
} hpacmlt_gradient;

#define HPACMLT_NORM_2 0
#define HPACMLT_NORM_MAX 1

typedef struct hpacmlt_gradients_s hpacmlt_gradients;

/* Lays out a set of n >= 0 gradients, whose memory stays the caller's, at the
 * same addresses while the set lives.  HPACML_E_ALIAS: a `to` overlaps another
 * tensor, or the same memory appears twice as `from` and `to`.  Synchronises
 * the device. */
hpacml_status hpacmlt_gradients_create(const hpacmlt_gradient *gradients, int64_t n, hpacmlt_gradients **out);

/* Frees a set.  NULL-safe.  Synchronise streams that use it first. */
void hpacmlt_gradients_destroy(hpacmlt_gradients *set);

/* Bytes of scratch of the two calls below. */
hpacml_status hpacmlt_gradients_scratch(const hpacmlt_gradients *set, size_t *bytes);

/* norm[0] = the gradients' common norm, rounded to fp32: HPACMLT_NORM_2, the
 * square root of the sum of all squares in 64-bit floating point, or
 * HPACMLT_NORM_MAX, the largest magnitude (NaN if there is a NaN).  No values:
 * 0. */
hpacml_status hpacmlt_gradients_norm(const hpacmlt_gradients *set, int32_t kind, float *norm, void *scratch,
                                     size_t scratch_bytes, void *stream);

/* The same, and each gradient times min(1, most / (norm + 1e-6)) (that factor
 * computed in 64 bits from the norm before its rounding, and rounded to fp32;
 * NaN if the norm is), the product in fp32, rounded to its `to` type.
 * most >= 0. */
hpacml_status hpacmlt_gradients_clip(const hpacmlt_gradients *set, int32_t kind, double most, float *norm,
                                     void *scratch, size_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HPACMLT_H */
