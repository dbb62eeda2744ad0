/*
 * mx_norm.h -- RMS norm with the residual's addition, delivered in the form that the
 * next product reads (an MX tensor, or 8 bits with a Float32 scale per 128), and its
 * gradients.  In the library of mx.h and by its conventions.
 *
 *     h    = x + residual, rounded to the tensors' type (h = x without a residual)
 *     rstd = 1 / sqrt(mean of h^2 over the row + eps)
 *     y    = h * weight * rstd in Float32 (weight NULL: 1)
 * Sums are Float32: a row whose sum of squares passes Float32's range has rstd 0 (and y
 * zero, or NaN where h or h * weight is infinite).  With eps = 0 a row of zeros, or of
 * numbers whose squares vanish in Float32, has rstd infinity, and its zeros give NaN.
 *
 * Common arguments
 *   x, ldx              [rows, cols] of type dt, rows ldx elements apart
 *   residual, ldr       the same, or NULL
 *   weight, w_dt        [cols] of type w_dt, or NULL
 *   eps                 finite, not negative (else MX_ERR_ENUM)
 *   h_out, ldh          receives h, or NULL; may be x or the residual itself, with
 *                       its pitch (the stream is then updated in place)
 *   y_out, ldy          receives y rounded to dt, or NULL; may be x or the residual
 *                       (with its pitch) where h_out is not
 *   rstd_out            [rows] Float32, or NULL (the backward pass wants it)
 * Tensor pointers are 16-byte aligned and pitches a multiple of 16 bytes, at least
 * cols (a pitch of an absent tensor is not looked at); rstd_out is 4-byte aligned.
 * MX_ERR_UNSUPPORTED: 2^31 rows and more, or 2^32 columns and more.
 */
#ifndef MX_NORM_H
#define MX_NORM_H

#include "mx_b128.h"

#ifdef __cplusplus
extern "C" {
#endif

/* No cast: y_out is required. */
int mx_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldr,
               const void *weight, mx_dtype_t w_dt, mx_dtype_t dt,
               int64_t rows, int64_t cols, float eps,
               void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out,
               void *hip_stream);

/* elems_out, scales_out receive, bit for bit, what mx_quantize (axis 1, fmt, rnd)
 * writes for the Float32 y: sizes mx_elem_bytes / mx_scale_bytes (axis 1).
 * rnd: not MX_ROUND_STOCHASTIC. */
int mx_rmsnorm_q(const void *x, int64_t ldx, const void *residual, int64_t ldr,
                 const void *weight, mx_dtype_t w_dt, mx_dtype_t dt,
                 int64_t rows, int64_t cols, float eps, mx_format_t fmt, mx_round_t rnd,
                 void *elems_out, uint8_t *scales_out,
                 void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out,
                 void *hip_stream);

/* ... what mx_quantize_b128 (axis 1, tile 0, fmt) writes for the Float32 y. */
int mx_rmsnorm_b128(const void *x, int64_t ldx, const void *residual, int64_t ldr,
                    const void *weight, mx_dtype_t w_dt, mx_dtype_t dt,
                    int64_t rows, int64_t cols, float eps, mx_format_t fmt,
                    void *elems_out, float *scales_out,
                    void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out,
                    void *hip_stream);

/*
 * Gradients of y with respect to h -- which x and the residual share -- and the
 * weight; a cast behind y passes its gradient through unchanged.  With
 * xhat = h * rstd and g = dy * weight:
 *     dx      = rstd * (g - xhat * mean of g xhat over the row) + dh
 *     dweight = sum over the rows of dy * xhat         (Float32, [cols])
 * dy, h, dh, dx: [rows, cols] of type dt with their pitches; dh (the gradient that
 * reaches h by other ways) may be NULL; dx may be dy, h or dh itself, with its
 * pitch.  rstd as the forward pass wrote it.  dweight may be NULL (not wanted; it is
 * written, not added to); it needs mx_rmsnorm_bwd_workspace_bytes bytes of scratch
 * memory, from the device's memory pool in stream order, or in the _ws form from
 * `workspace` (16-byte aligned; too small: MX_ERR_WORKSPACE; NULL: as the plain
 * form).  The order of every sum depends on the shape alone.  rows = 0 with a
 * dweight writes zeros.
 * While hip_stream is captured, memory from the pool becomes an allocation and a
 * release inside the graph, and what two graphs that run at the same time get is for
 * the runtime to say: such graphs want the _ws form with a workspace each, which
 * has to stay theirs for as long as they are replayed.
 */
size_t mx_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t cols);
int mx_rmsnorm_bwd(const void *dy, int64_t lddy, const void *h, int64_t ldh,
                   const void *weight, mx_dtype_t w_dt, const float *rstd,
                   const void *dh, int64_t lddh, mx_dtype_t dt, int64_t rows, int64_t cols,
                   void *dx, int64_t lddx, float *dweight, void *hip_stream);
int mx_rmsnorm_bwd_ws(const void *dy, int64_t lddy, const void *h, int64_t ldh,
                      const void *weight, mx_dtype_t w_dt, const float *rstd,
                      const void *dh, int64_t lddh, mx_dtype_t dt, int64_t rows, int64_t cols,
                      void *dx, int64_t lddx, float *dweight,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
