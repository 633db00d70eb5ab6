/* hh_mx.h -- C ABI of the residual path of a layer (dropout, the residual's addition, root-mean-square norm) and of products in
 * microscaled 8- and 4-bit floating point, forward and backward.
 *
 * A pre-norm layer is a chain of   h = x + dropout(b),  xn = rmsnorm(h; g),  b' = xn W^T   (hh.h).  Here each link is an operator of its
 * own, for parts of a model that hh_layer_fwd does not hold (a final norm, a projection of its own, a branch that is dropped in training),
 * and the product takes operands of 8 or 4 bits: half and a quarter of bfloat16's memory, and on the matrix cores up to twice (where the caller allows
 * sums of fewer bits) and four times its rate:
 *
 *     hh_add_norm_fwd (packed xn) -> hh_mx_product -> hh_dropout or the next hh_add_norm_fwd
 *     backward:  hh_mx_quantise of dy by row and by column -> hh_mx_product for dx (with W packed by column) and for dW (with xn packed
 *                by column) -> hh_add_norm_bwd
 *
 * The general rules of hh.h hold: statuses and hh_last_error(), device pointers of 16-byte alignment, buffers that the caller owns, work
 * enqueued on `stream` without synchronisation, allocation or copies, checks of arguments before any of it.  The context's device has to
 * be the calling thread's current one (HH_ERR_INVALID_ARG otherwise).  Every result is the same from run to run, bit for bit;
 * a row's sums may be added in another order in a call with another number of rows.  Two calls that may run at the same time need a workspace each.
 */
#ifndef HH_MX_H
#define HH_MX_H

#include "hh.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Dropout.  Element (row, column) is kept where its 16 random bits are at least t = p 65536 rounded, and then multiplied by
 * 65536 / (65536 - t), so that its expectation is unchanged; otherwise it is 0, whatever it held (NaN too).  The mask is never stored:
 * a gradient is dropped by the same call with the same numbers.
 *
 * The bits are those of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011) with the seed as
 * its key and the counter (column / 8, row, offset mod 2^32, offset / 2^32): word (column mod 8) / 2 of the result, its low half for even columns.
 * They depend on nothing else: not on strides, types, the sizes of the launch or on what else the tensor holds.
 *
 * offset numbers the uses of a seed: a layer, a micro-batch and a step each have one of their own.  step (device, may be NULL) is added to it
 * when the kernel runs: a captured graph that advances *step between its replays drops other elements in each of them. */
typedef struct {
    uint64_t seed, offset;
    const uint64_t *step;  /* device, 8-byte aligned, or NULL */
    double p;              /* share that is dropped, 0 .. 1 */
} hh_dropout_cfg;

/* y = dropout(x), [rows, cols] of dtype, rows ldx and ldy elements apart.  y may be x (ldy = ldx then).  Here and below, rows times
 * columns / 8, rounded up, are below 2^31 (HH_ERR_UNSUPPORTED_SHAPE otherwise; columns as padded, where a tensor is packed). */
int hh_dropout(hh_ctx *ctx, const hh_dropout_cfg *drop, int64_t rows, int64_t cols, int32_t dtype, const void *x, int64_t ldx,
               void *y, int64_t ldy, void *stream);

/* Microscaled formats (OCP Microscaling Formats 1.0, MXFP8 E4M3 and MXFP4 E2M1).  The values of a row of k are taken in blocks of 32; a
 * block has a scale X = 2^e, e = max(floor(log2 m) - E, -127) with m its largest magnitude and E the exponent of the format's largest
 * number (8: 448, 2: 6), and each value v is held as the number of the format nearest to v / X, the even one of two, the largest one where
 * v / X is past it.  A block that holds a NaN or an infinity has the scale NaN and stands for NaNs.
 *
 * In memory: codes [rows, K] with K = k rounded up to a multiple of 256 (HH_MX_PAD), a byte each (E4M3) or half a byte (E2M1, the even
 * value in the low four bits); scales [rows, K / 32], a byte each, e + 127, 255 for NaN.  What is past k is zeros, codes and scales, and every
 * call that reads a packed tensor relies on it.  Both pointers are 16-byte aligned. */
typedef enum { HH_MX_NONE = 0, HH_MX_E4M3 = 1, HH_MX_E2M1 = 2 } hh_mx_format;
#define HH_MX_PAD 256
typedef struct {
    void *codes;
    uint8_t *scales;
} hh_mx_tensor;

/* Bytes of a packed tensor of `rows` rows of k values.  Either pointer may be NULL. */
int hh_mx_sizes(int32_t format, int64_t rows, int64_t k, size_t *codes_bytes, size_t *scales_bytes);

/* x [rows, cols] of dtype, rows ldx elements apart, packed by row ([rows, cols], blocks along a row) and by column (the transposed
 * copy [cols, rows], blocks along a column of x), each where it is not NULL; both take one read of x. */
int hh_mx_quantise(hh_ctx *ctx, int64_t rows, int64_t cols, int32_t dtype, const void *x, int64_t ldx, int32_t format,
                   const hh_mx_tensor *by_row, const hh_mx_tensor *by_column, void *stream);

/* The values [rows, k] that a packed tensor stands for, in dtype, rows ldy elements apart.  bfloat16 holds them exactly under the scale bytes 3 to
 * 246 (E4M3) and up to 252 (E2M1).  Packing writes no larger ones, and smaller ones for blocks below 2^-116 alone.  Outside of that a value
 * below 2^-130 may lie between two multiples of 2^-133, of which it becomes the nearest one, and one from 2^128 on, which fp32 does not hold
 * either, becomes an infinity. */
int hh_mx_values(hh_ctx *ctx, int64_t rows, int64_t k, int32_t format, const hh_mx_tensor *q, int32_t dtype, void *y, int64_t ldy,
                 void *stream);

/* Residual addition and norm:
 *     h = x + dropout(b)  rounded to dtype,   xn = h g / sqrt(mean(h^2) + eps)
 * x, b, h, xn: [rows, hidden] contiguous; g: [hidden]; all of dtype, arithmetic in fp32, a row's sum and root in 64 bits from eight values on.  b NULL: h is x, which is not
 * written again (h has to be NULL).  h may be x or b.  xn is written where it is not NULL; q receives xn, before it is rounded,
 * packed in `format` (HH_MX_NONE: q has to be NULL).  One of xn and q at least.  drop NULL: nothing is dropped. */
typedef struct {
    int32_t rows, hidden;  /* hidden: 1 .. 32768; rows: 1 .. 2^24, 2^34 values at most */
    float eps;             /* inside the square root, >= 0 */
    int32_t dtype;         /* hh_dtype */
    int32_t format;        /* hh_mx_format of q */
} hh_add_norm_cfg;
int hh_add_norm_fwd(hh_ctx *ctx, const hh_add_norm_cfg *cfg, const hh_dropout_cfg *drop, const void *x, const void *b, const void *g,
                    void *h, void *xn, const hh_mx_tensor *q, void *stream);

/* Gradients, from the h of the forward call (x where there was no branch), the gradient dxn of xn (the packed copy passes its gradient
 * on as if it were xn) and, where it is not NULL, the gradient dh that reaches h from elsewhere:
 *     u = dxn g,  r = 1 / sqrt(mean(h^2) + eps):   dx = dh + r (u - h r^2 mean(u h)),   db = dropout(dx),   dg (+)= sum over rows of dxn h r
 * db is of the dx that has not been rounded; NULL: it is not written (without dropout it is dx).  dg: [hidden] fp32, added to where
 * accumulate != 0; NULL: not wanted.  dx may be dh, dxn or h, and db any other one of them.  workspace of hh_add_norm_sizes bytes (only used for dg). */
int hh_add_norm_sizes(const hh_add_norm_cfg *cfg, size_t *workspace_bytes);
int hh_add_norm_bwd(hh_ctx *ctx, const hh_add_norm_cfg *cfg, const hh_dropout_cfg *drop, const void *h, const void *g, const void *dxn,
                    const void *dh, void *dx, void *db, float *dg, int accumulate, void *workspace, void *stream);

/* c [m, n] (=|+=) a b^T of two packed tensors a [m, k] and b [n, k], formats in any combination; c of dtype, rows ldc elements apart,
 * sums in fp32, rounded once (with accumulate: old value and sum are added in fp32 first).
 *
 * HH_MX_SUMS_F32 (0): every product of two values enters a sum of fp32.  With an E4M3 operand on either side both are widened to bfloat16 with
 * their scales (as hh_mx_values does: exactly but at the ends of its range) and multiplied at that type's rate; E2M1 on both sides runs at its own, at
 * which nothing is lost.
 *
 * HH_MX_SUMS_FAST allows fewer bits where they make a call faster, which they do into HH_BF16 with an E4M3 operand and more than 32 rows: the
 * matrix cores' instruction for it, of twice bfloat16's rate, aligns the 64 products that it adds to the largest of them and keeps a little more
 * than 16 bits there (E4M3 on both sides; some two more with E2M1 on one).  Against exact sums that leaves 1.5e-5 of a result's size for normal values and
 * 1e-4 with outliers of 30 to 100 times among them, next to the 2^-8 that rounding to bfloat16 leaves at most.
 *
 * A packed operand is below 2^32 - 2^25 bytes, c at most 2^33 elements.  workspace of hh_mx_product_sizes bytes (128 MiB at most), NULL where that is 0. */
typedef enum { HH_MX_SUMS_F32 = 0, HH_MX_SUMS_FAST = 1 } hh_mx_sums;
typedef struct {
    int32_t m, n, k;
    int32_t a_format, b_format;
    int32_t dtype;
    int64_t ldc;
    int32_t sums;  /* hh_mx_sums */
} hh_mx_product_cfg;
int hh_mx_product_sizes(const hh_mx_product_cfg *cfg, size_t *workspace_bytes);
int hh_mx_product(hh_ctx *ctx, const hh_mx_product_cfg *cfg, const hh_mx_tensor *a, const hh_mx_tensor *b, void *c, int accumulate,
                  void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HH_MX_H */
