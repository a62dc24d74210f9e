/*
 * hpacml8.h -- dense layers in 8 bits, the companion of hpacml.h: answering
 * with a surrogate's layers in 8-bit integers, and learning one from collected
 * samples with the activations kept in 8 bits.
 *
 * Conventions are those of hpacml.h: device pointers on the current HIP
 * device, a hipStream_t passed as void*, statuses instead of exceptions, every
 * check done on the host before anything is enqueued.  A matrix is row-major
 * with a row pitch in elements (a pitch may exceed the width: rows inside a
 * wider record); a row is a point of the sweep.  The library verifies that
 * every operand is device memory of the current device and lies inside its
 * allocation (HPACML_E_INVAL, HPACML_E_RANGE), and that nothing written
 * overlaps another operand (HPACML_E_ALIAS; rows of one record with equal
 * pitches may interleave).  Calls allocate nothing; what they need beyond
 * their operands is scratch memory of the caller, whose contents mean nothing
 * between calls.  No call synchronises, except the creation of a layer; none
 * uses atomic operations: equal calls give equal bits.  Calls with scratch,
 * operands and outputs of their own may overlap on different streams.
 */
#ifndef HPACML8_H
#define HPACML8_H

#include "hpacml.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HPACML8_MAX_WIDTH 16384   /* inputs and outputs of a layer */
#define HPACML8_BLOCK 32          /* channels of a row that share one exponent */

/* ---- y = act(x W^T + b) in 8-bit integers ---------------------------------
 * Each row x_i of the inputs and each row W_j of the weights is rounded to
 * codes -127..127 with a scale of its own:
 *     s_i = max_k |x_ik| / 127,  q_ik = rint(x_ik * (127 / max_k |x_ik|))
 * (fp32 arithmetic, ties to even), t_j and w_jk the same of W_j, and
 *     y_ij = act(s_i * t_j * sum_k q_ik w_jk + b_j),
 * the sum in exact 32-bit integers, the rest in fp32 (what lies between the sum
 * and the result leaves fp32's range only where the result does), rounded once
 * to y's type.  A row whose largest magnitude is below 2^-119 counts as zeros; a row
 * of inputs or weights that holds an infinity or a NaN makes the results it
 * reaches NaN (a ReLU keeps a NaN). */
typedef struct hpacml8_linear_s hpacml8_linear;

/* Lays a layer's weights out in device memory.
 *   W: fp32 [n_out][n_in], b: fp32 [n_out] or NULL (no bias); HOST or DEVICE
 *   memory, copied (beyond its allocation on the device: HPACML_E_RANGE).
 *   n_in, n_out: 1..HPACML8_MAX_WIDTH (above: HPACML_E_UNSUPPORTED).
 * Synchronises the device (also before it reads W). */
hpacml_status hpacml8_linear_create(int32_t n_in, int32_t n_out, const float *W, const float *b,
                                    hpacml8_linear **out);

/* Frees a layer.  NULL-safe.  Synchronise streams that use it first. */
void hpacml8_linear_destroy(hpacml8_linear *layer);

/* Bytes of scratch hpacml8_linear_run needs for n_rows rows (never shrinking
 * with n_rows; 0 for no rows). */
hpacml_status hpacml8_linear_scratch(const hpacml8_linear *layer, int64_t n_rows, size_t *bytes);

/* y [n_rows][n_out] from x [n_rows][n_in].
 *   x_dtype, y_dtype: HPACML_F32 or HPACML_BF16; ldx >= n_in, ldy >= n_out;
 *   act: HPACML_ACT_*; scratch: 16-byte aligned, `scratch_bytes` at least what
 *   hpacml8_linear_scratch says (HPACML_E_RANGE otherwise).
 * Pointers are aligned to their type.  Zero rows: HPACML_OK, nothing
 * launched.  Asynchronous on `stream`. */
hpacml_status hpacml8_linear_run(const hpacml8_linear *layer, const void *x, int32_t x_dtype, int64_t ldx,
                                 int64_t n_rows, void *y, int32_t y_dtype, int64_t ldy, int32_t act, void *scratch,
                                 size_t scratch_bytes, void *stream);

/* ---- activations kept in 8 bits -------------------------------------------
 * What a layer's backward pass needs of its input a, at a little over half of
 * bf16's memory.  HPACML8_BLOCK channels of a row share a power of two 2^e:
 *   after a ReLU (act HPACML_ACT_RELU): a / 2^e rounded to codes 0..255, e the
 *     smallest with max a < 2^(e + 8); a positive a keeps at least code 1, so
 *     code 0 says exactly where the ReLU let nothing through;
 *   otherwise (HPACML_ACT_IDENTITY): codes -127..127, stored plus 128, e the
 *     smallest with max |a| < 2^(e + 7).
 * (Ties to even; what would round beyond the largest code is cut to it; e is
 * at least -126.)  A code times its power of two is exact in bf16.  A block
 * with an infinity or a NaN has exponent byte 255 and stands for values that
 * are all infinite or NaN.  After a ReLU a NaN has code 0: the backward pass
 * lets nothing through there. */
typedef struct {
    void *codes;          /* DEVICE, one byte each: [rows][ld_codes], 16-byte aligned */
    void *exps;           /* DEVICE, one byte each: [rows][ld_exps], e + 127 per block */
    int64_t rows;         /* >= 0 */
    int64_t ld_codes;     /* a multiple of 32, at least width */
    int64_t ld_exps;      /* at least ceil(width / 32) */
    int32_t width;        /* channels, 1..HPACML8_MAX_WIDTH */
    int32_t act;          /* HPACML_ACT_*: what the activation is the output of */
} hpacml8_checkpoint;

/* Keeps act(z) in `c`, and writes it, rounded to its type, to `a` as well
 * where `a` is not NULL.
 *   z [rows][width], a [rows][width]: types HPACML_F32 or HPACML_BF16, ldz,
 *   lda >= width; `a` may be z itself (same pointer, type and pitch).
 * The codes of the channels that fill up the last block are written too (they
 * stand for 0).  Asynchronous on `stream`. */
hpacml_status hpacml8_checkpoint_save(const hpacml8_checkpoint *c, const void *z, int32_t z_dtype, int64_t ldz,
                                      void *a, int32_t a_dtype, int64_t lda, void *stream);

/* What `c` stands for, as a [rows][width] of type HPACML_F32 or HPACML_BF16
 * (exact in both).  Asynchronous on `stream`. */
hpacml_status hpacml8_checkpoint_load(const hpacml8_checkpoint *c, void *a, int32_t a_dtype, int64_t lda,
                                      void *stream);

/* ---- a linear layer's backward pass from its kept input -------------------
 * The layer y = a W^T + b with `a` kept in `c` (n_in = c->width), dy the
 * gradient of y:
 *     dw[j][k] (+)= sum_i dy_ij a_ik      db[j] (+)= sum_i dy_ij
 *     dx[i][k]  =  sum_j dy_ij W_jk where c lets it through, else 0
 * (c lets through where its code is not 0 after a ReLU, everywhere else).
 *   dtype: HPACML_F32 or HPACML_BF16, the type of dy [rows][n_out], W
 *   [n_out][n_in] and dx [rows][n_in]; dw [n_out][n_in] and db [n_out] are
 *   fp32.  Any of dw, db, dx may be NULL (not wanted; W is read for dx only).
 *   accumulate: nonzero adds to dw and db (batches in parts), zero sets them.
 *   n_out: 1..HPACML8_MAX_WIDTH.
 * bf16: products of exact bf16 values on the matrix cores, fp32 sums; dx
 * rounded once.  fp32: each fp32 operand is the exact sum of three bf16 terms
 * (below 2^-110: to within 2^-134, so that less than that counts as 0); dw takes
 * all three products, dx the six largest of nine (what is left out is below
 * 2^-23 of a product).  Infinities and NaNs in dy and W give what the sums above
 * give; so do those that `c` stands for in bf16, while in fp32 a block of `c`
 * with exponent byte 255 counts as NaN in dw.
 * Zero rows: dw and db are set to 0 (accumulate: left).  Asynchronous on
 * `stream`. */
hpacml_status hpacml8_backward(const hpacml8_checkpoint *c, const void *dy, int32_t dtype, int64_t lddy,
                               int32_t n_out, const void *W, int64_t ldw, float *dw, int64_t lddw, float *db,
                               void *dx, int64_t lddx, int32_t accumulate, void *scratch, size_t scratch_bytes,
                               void *stream);

/* Bytes of scratch (16-byte aligned) hpacml8_backward needs for these
 * operands; want_dw (dw or db) and want_dx say which of its outputs are
 * wanted.  With many rows a dy is read in place if it is bf16, its pointer
 * 16-byte aligned, lddy a multiple of 8 (below 2^22) and n_out one of 32 (of 8
 * where dx is not wanted); any other is first laid out in the scratch memory.
 * A smaller number of rows may need more: ask for each. */
hpacml_status hpacml8_backward_scratch(const hpacml8_checkpoint *c, const void *dy, int32_t dtype, int64_t lddy,
                                       int32_t n_out, int32_t want_dw, int32_t want_dx, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* HPACML8_H */
