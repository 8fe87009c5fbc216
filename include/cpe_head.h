/*
 * cpe_head.h -- C ABI of the operators that lead to the decoder's input: the
 * pixel head of the network whose output cpe_decode reads.  Group norm with
 * an activation over channels-last maps, and the matrix product with bias,
 * activation and residual that projects a map's features to its embedding
 * (or a block's features to the next one's), each with its gradient.
 *
 * Types.  Maps and weight matrices have the handle's dtype (f32, f16 or bf16; the
 * decoder reads the first two); per-channel vectors (gamma, beta, bias, their gradients) and
 * group statistics are float.  Sums, statistics and activations are formed in
 * binary32 and each output is rounded once, to nearest even; where a product's
 * operand is an intermediate result, its entry says how it is held.
 *
 * Activations of u:  CPE_ACT_NONE u;  CPE_ACT_RELU max(u, 0) (derivative 0 at
 * 0);  CPE_ACT_SILU u / (1 + e^-u);  CPE_ACT_GELU u (1 + erf(u / sqrt 2)) / 2.
 * NaNs propagate, through the derivatives as well; SiLU and GELU of -infinity
 * are NaN (-inf * 0), and so are their derivatives at either infinity.
 *
 * Layouts.  Row-major; a row's elements (channels, features) are contiguous,
 * and rows are a stride apart that counts elements.  Pointers need their
 * element's alignment only; rows whose pointers and strides are 16-byte
 * aligned are faster in the products.  Strides are given per call and must be
 * at least the row length; sample strides must keep the samples apart.
 *
 * Ownership.  The caller owns every buffer passed to a call (device memory).
 * The handle owns the scratch, allocated at create and freed at destroy; the
 * calls themselves never allocate, never synchronise and never copy to the
 * host: they enqueue work on `stream`.  Nothing is kept from one call for the
 * next, and results do not vary from run to run (sums have a fixed order).
 *
 * Errors.  Argument errors are found on the host before any work is enqueued
 * and return CPE_ERR_INVALID_ARG; a failed launch returns CPE_ERR_HIP (the
 * call's outputs are then undefined, later calls are unaffected).
 *
 * Graphs and threads.  Calls may be captured into HIP graphs (the handle must
 * outlive them).  A handle may be used by one stream at a time, on the device
 * that was current when it was created.
 */
#ifndef CPE_HEAD_H
#define CPE_HEAD_H

#include "cpe_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* (f32 and f16 have the codes of cpe_dtype) */
typedef enum { CPE_HEAD_F32 = 0, CPE_HEAD_F16 = 1, CPE_HEAD_BF16 = 2 } cpe_head_dtype;

typedef enum { CPE_ACT_NONE = 0, CPE_ACT_RELU = 1, CPE_ACT_SILU = 2, CPE_ACT_GELU = 3 } cpe_activation;

typedef struct cpe_norm cpe_norm;
typedef struct cpe_linear cpe_linear;

/*
 * Group norm with an activation, channels last.  For sample b, group g of the
 * C / G channels c with floor(c / (C / G)) = g, over its n = P_b C / G values:
 *   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps),
 *   u = (x - mean) rstd gamma_c + beta_c,  y = act(u).
 * P_b is the sample's number of pixels: `pixels`, or valid[b] of them where
 * `valid` is given (clamped to 0 .. pixels).  Pixels from P_b on are not read,
 * their outputs are 0.  A sample without pixels has mean 0, rstd 1/sqrt(eps).
 *   out           receives the handle (NULL on failure)
 *   max_samples   1..65535 samples of a call at most
 *   max_pixels    1..2^31 - 2^23 pixels of a sample at most
 *   channels      1..8192, groups: a divisor of it
 *   eps           finite, > 0
 */
cpe_status cpe_norm_create(cpe_norm **out, int32_t max_samples, int32_t max_pixels, int32_t channels,
                           int32_t groups, cpe_head_dtype dtype, cpe_activation act, float eps);

/*
 * y = act(norm(x)), asynchronously on `stream`.
 *   samples, pixels   0 .. the handle's maxima; either 0 enqueues nothing
 *   x, y              [samples][pixels][C], pixel stride x_ld / y_ld,
 *                     sample stride x_sample / y_sample (elements).  y may be x
 *                     itself with the same strides; otherwise they may not overlap
 *   gamma, beta       device [C] float, or NULL: 1, 0
 *   valid             device [samples] int32, or NULL
 *   stats             device [samples][G][2] float: mean and rstd for the
 *                     gradient, or NULL
 */
cpe_status cpe_norm_forward(cpe_norm *h, hipStream_t stream, int32_t samples, int32_t pixels, const void *x,
                            int64_t x_ld, int64_t x_sample, const float *gamma, const float *beta,
                            const int32_t *valid, void *y, int64_t y_ld, int64_t y_sample, float *stats);

/*
 * Gradient of cpe_norm_forward, from x, dy and the forward's stats:
 *   du = dy act'(u);  dbeta_c = sum du;  dgamma_c = sum du xh, xh = (x - mean) rstd;
 *   dx = rstd (gamma_c du - (a + xh q) / n), a and q the group's sums of
 *   gamma_c du and gamma_c du xh.
 * dx, dgamma, dbeta: any may be NULL (not wanted), not all.  dx may be dy or
 * x itself with the same strides.  dgamma and dbeta are written, not added to,
 * and sum over the samples; with samples or pixels 0 they are 0, and all three
 * may be NULL.
 */
cpe_status cpe_norm_backward(cpe_norm *h, hipStream_t stream, int32_t samples, int32_t pixels, const void *x,
                             int64_t x_ld, int64_t x_sample, const void *dy, int64_t dy_ld, int64_t dy_sample,
                             const float *gamma, const float *beta, const int32_t *valid, const float *stats,
                             void *dx, int64_t dx_ld, int64_t dx_sample, float *dgamma, float *dbeta);

cpe_status cpe_norm_destroy(cpe_norm *h);

/* Bytes of device memory the handle holds (0 for NULL). */
size_t cpe_norm_workspace_bytes(const cpe_norm *h);

/*
 * Matrix product with an epilogue: z = x w^T + bias, y = act(z) + residual.
 *   max_rows       1..2^31 - 2^23 rows (pixels, tokens) of a call at most
 *   in_features    K, 1..65536; out_features N, 1..65536
 * The handle's scratch is what calls of up to max_rows rows can use: up to
 * 32 MiB for products split along k and their gradients' partial sums, up to 8
 * MiB for those of dbias, and, with an activation, max_rows x N of the dtype for
 * dz where the gradient is neither one of few rows (up to 64) nor, in 16 bits,
 * narrow (N and K multiples of 8, up to 128 x 256 or 64 x 512).
 */
cpe_status cpe_linear_create(cpe_linear **out, int32_t max_rows, int32_t in_features, int32_t out_features,
                             cpe_head_dtype dtype, cpe_activation act);

/*
 * y [rows][N] from x [rows][K] and w [N][K], asynchronously on `stream`.
 *   rows        0 .. the handle's maximum; 0 enqueues nothing
 *   x_ld, w_ld, y_ld, residual_ld, preact_ld   row strides in elements
 *   bias        device [N] float or NULL
 *   residual    device [rows][N] or NULL; may be y itself with the same stride
 *   preact      device [rows][N] or NULL: receives z for the gradient
 * Apart from that residual, y and preact overlap no input and not each other.
 */
cpe_status cpe_linear_forward(cpe_linear *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                              const void *w, int64_t w_ld, const float *bias, const void *residual,
                              int64_t residual_ld, void *y, int64_t y_ld, void *preact, int64_t preact_ld);

/*
 * Gradient of cpe_linear_forward, from x, w, dy and the forward's preact:
 *   dz = dy act'(z);  dx = dz w;  dw = dz^T x;  dbias = sum over rows of dz.
 * (The residual's gradient is dy.)  preact may be NULL for CPE_ACT_NONE only.
 * dx [rows][K], dw [N][K], dbias [N] float: any may be NULL, not all; they
 * are written, not added to, and overlap no input; with rows 0, dw and dbias
 * are 0, and all three may be NULL.  The products take dz rounded to the dtype,
 * as their operand (in f16 a |dz| beyond 65504, which takes a |dy| beyond 57,000,
 * becomes an infinity); dbias sums it unrounded.
 */
cpe_status cpe_linear_backward(cpe_linear *h, hipStream_t stream, int32_t rows, const void *x, int64_t x_ld,
                               const void *w, int64_t w_ld, const void *dy, int64_t dy_ld, const void *preact,
                               int64_t preact_ld, void *dx, int64_t dx_ld, void *dw, int64_t dw_ld, float *dbias);

cpe_status cpe_linear_destroy(cpe_linear *h);

/* Bytes of device memory the handle holds (0 for NULL). */
size_t cpe_linear_workspace_bytes(const cpe_linear *h);

#ifdef __cplusplus
}
#endif
#endif /* CPE_HEAD_H */
