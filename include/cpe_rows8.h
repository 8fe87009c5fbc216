/*
 * cpe_rows8.h -- C ABI of the operators on rows held in 8 bits: rows packed
 * and unpacked, RMS norm with the residual's addition that writes them, the
 * integer matrix product that reads them, and gradients from checkpoints in
 * them.  Types, layouts, ownership, errors, graphs and threads are those of
 * cpe_head.h.
 *
 * Rows in 8 bits.  Row r is `width` signed bytes q and one float, its scale s:
 * it stands for the values q s.  A row x is packed with m = max |x|,
 *   s = max(m / 127, 2^-126),  q = rint(x / s)     (|q| <= 127),
 * both quotients rounded to binary32, ties of rint to even.  A row that holds a
 * NaN or an infinity has scale NaN and q = 0: all its values are NaN.  Byte rows
 * are a stride apart that counts bytes and need no alignment; those whose
 * pointers and strides are 16-byte aligned are faster in the products.
 */
#ifndef CPE_ROWS8_H
#define CPE_ROWS8_H

#include "cpe_head.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cpe_rms cpe_rms;
typedef struct cpe_linear8 cpe_linear8;

/*
 * Packs x [rows][width] into q and scale [rows], asynchronously on `stream`
 * (of the current device).
 *   rows    0 .. 2^31 - 2^23; 0 enqueues nothing
 *   width   1 .. 65536
 * q and scale overlap neither x nor each other.
 */
cpe_status cpe_rows8_pack(hipStream_t stream, int32_t rows, int32_t width, cpe_head_dtype dtype, const void *x,
                          int64_t x_ld, int8_t *q, int64_t q_ld, float *scale);

/* x = q s, a binary32 product rounded to the dtype; sizes as above.  x overlaps neither input. */
cpe_status cpe_rows8_unpack(hipStream_t stream, int32_t rows, int32_t width, const int8_t *q, int64_t q_ld,
                            const float *scale, cpe_head_dtype dtype, void *x, int64_t x_ld);

/*
 * RMS norm over the channels of each row (pixel, token), with the addition of
 * the residual stream before it:
 *   h = x, or x + residual rounded to the dtype;
 *   rstd = 1 / sqrt(sum_c h_c^2 / C + eps),  y_c = h_c rstd gamma_c.
 * The sum of squares is binary32's: where it passes 3.4e38, rstd is 0 (as it is
 * for a row that holds an infinity, whose own y is then a NaN).
 *   out        receives the handle (NULL on failure)
 *   max_rows   1..2^31 - 2^23 rows of a call at most
 *   channels   C, 1..16384
 *   eps        finite, 2^-126 or more
 * The handle's scratch are the partial sums of dgamma: up to 8 MiB, or 256 x C
 * floats where that is more.
 */
cpe_status cpe_rms_create(cpe_rms **out, int32_t max_rows, int32_t channels, cpe_head_dtype dtype, float eps);

/*
 * The norm of x [rows][C], asynchronously on `stream`.
 *   rows       0 .. the handle's maximum; 0 enqueues nothing
 *   residual   device [rows][C] or NULL
 *   gamma      device [C] float, or NULL: 1
 *   sum        device [rows][C] or NULL: receives h
 *   y          device [rows][C] or NULL: receives y
 *   q, scale   device rows in 8 bits, or both NULL: receive y, packed before it
 *              is rounded to the dtype
 *   rstd       device [rows] float, or NULL: for the gradient
 * One of sum, y and q is given at least.  sum and y may each be x or residual
 * with the same stride; apart from that no output overlaps an input or another
 * output.
 */
cpe_status cpe_rms_forward(cpe_rms *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                           const void *residual, int64_t residual_ld, const float *gamma, void *sum, int64_t sum_ld,
                           void *y, int64_t y_ld, int8_t *q, int64_t q_ld, float *scale, float *rstd);

/*
 * Gradient of cpe_rms_forward, from h, dy and the forward's rstd:
 *   t = dy gamma,  xh = h rstd,  a = sum_c t xh / C;
 *   dx = rstd (t - xh a) + dsum;   dgamma_c = sum over rows of dy xh.
 * dx is the gradient of x and of the residual.
 *   h_rows, h_scale   h [rows][C] of the dtype and NULL, or h in 8 bits
 *                     (strides then count bytes) and its scales
 *   dsum              device [rows][C] or NULL: the gradient that reaches h
 *                     past the norm
 * dx [rows][C], dgamma [C] float: either may be NULL, not both.  dx may be dy,
 * dsum or (not in 8 bits) h_rows with the same stride; otherwise they overlap
 * no input.  dgamma is written, not added to; with rows 0 it is 0, and both may
 * be NULL.
 */
cpe_status cpe_rms_backward(cpe_rms *h, hipStream_t stream, int32_t rows, const void *h_rows, int64_t h_ld,
                            const float *h_scale, const void *dy, int64_t dy_ld, const float *gamma,
                            const float *rstd, const void *dsum, int64_t dsum_ld, void *dx, int64_t dx_ld,
                            float *dgamma);

cpe_status cpe_rms_destroy(cpe_rms *h);

/* Bytes of device memory the handle holds (0 for NULL). */
size_t cpe_rms_workspace_bytes(const cpe_rms *h);

/*
 * Integer matrix product with an epilogue: rows q with scales s (a scale per
 * token), weight rows w with scales t (a scale per output channel),
 *   z_rn = (sum_k q_rk w_nk) s_r t_n + bias_n,  y = act(z) + residual.
 * The sum is an exact whole number (every signed byte is allowed), which is
 * then rounded to binary32; y and residual have the handle's dtype.
 *   max_rows       1..2^31 - 2^23 rows (pixels, tokens) of a call at most
 *   in_features    K, 1..65536; out_features N, 1..65536
 * The handle's scratch are the partial sums of products split along k: up to
 * 32 MiB.
 */
cpe_status cpe_linear8_create(cpe_linear8 **out, int32_t max_rows, int32_t in_features, int32_t out_features,
                              cpe_head_dtype dtype, cpe_activation act);

/*
 * y [rows][N] from q [rows][K], scale [rows], w [N][K] and w_scale [N],
 * asynchronously on `stream`; the other arguments are those of
 * cpe_linear_forward.
 */
cpe_status cpe_linear8_forward(cpe_linear8 *h, hipStream_t stream, int32_t rows, const int8_t *q, int64_t q_ld,
                               const float *scale, const int8_t *w, int64_t w_ld, const float *w_scale,
                               const float *bias, const void *residual, int64_t residual_ld, void *y, int64_t y_ld,
                               void *preact, int64_t preact_ld);

cpe_status cpe_linear8_destroy(cpe_linear8 *h);

/* Bytes of device memory the handle holds (0 for NULL). */
size_t cpe_linear8_workspace_bytes(const cpe_linear8 *h);

/*
 * cpe_linear_backward from a checkpoint in 8 bits: x = q scale, and (with an
 * activation) preact = zq z_scale, are rows in 8 bits; w, dy, the outputs and
 * the rest are those of cpe_linear_backward, on the same handle.  The gradient
 * of an integer product whose weights are kept in the dtype as well is this
 * one, too.
 *
 * dbias sums dz = dy act'(preact) unrounded.  The products take operands of the
 * dtype, one of which holds a rounding: x, where dz is dy or 0; dz, with the
 * mantissa of the row's scale (1 <= f < 2) as a factor, where the activation is
 * SiLU or GELU (x is then q times a power of two, and dx is divided by the
 * factor; in f16 a |dz| f beyond 65504 becomes an infinity).  In f16 values of
 * x below 2^-14 are subnormal, as x itself would be.
 */
cpe_status cpe_linear_backward8(cpe_linear *h, hipStream_t stream, int32_t rows, const int8_t *q, int64_t q_ld,
                                const float *scale, const void *w, int64_t w_ld, const void *dy, int64_t dy_ld,
                                const int8_t *zq, int64_t zq_ld, const float *z_scale, void *dx, int64_t dx_ld,
                                void *dw, int64_t dw_ld, float *dbias);

#ifdef __cplusplus
}
#endif
#endif /* CPE_ROWS8_H */
