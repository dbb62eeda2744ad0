/*
 * mx_b128.h -- 8-bit floating point with one Float32 scale for each block of 128
 * elements: the cast, its inverse and the matrix product, in the library of mx.h
 * and by its conventions (device pointers owned by the caller, asynchronous work
 * on hip_stream, mx_status_t results, argument errors found before anything is
 * launched, zero-sized problems a no-op).  Nothing here allocates.
 *
 * Where an MX block is 32 elements with a power-of-two scale, this form has
 *   1 x 128    blocks along a line (activations, gradients), or
 *   128 x 128  tiles (weights: the cast of the transpose is the transpose of the cast).
 * Formats are MX_FP8_E4M3 and MX_FP8_E5M2; anything else is MX_ERR_ENUM.
 *
 * Storage.  For a logical [R][L] tensor blocked along L, two separate arrays:
 *     elems  uint8 [R][128 * ceil(L/128)]    one element a byte; the fill of a
 *                                            partial last block is zero
 *     scales float [R][ceil(L/128)]          1 x 128
 *            float [ceil(R/128)][ceil(L/128)] 128 x 128
 * An element stands for elems * scales.
 */
#ifndef MX_B128_H
#define MX_B128_H

#include "mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the elems array, and number of Float32 scales, for a [rows, cols]
 * tensor cast along axis (tile: 0 = 1 x 128, 1 = 128 x 128); 0 for arguments out
 * of range. */
size_t mx_b128_elem_bytes(int64_t rows, int64_t cols, int axis);
size_t mx_b128_scale_count(int64_t rows, int64_t cols, int axis, int tile);

/*
 * The cast.  src, src_dt, rows, cols, ld as mx_quantize.  axis = 1: blocks along
 * the rows, R = rows and L = cols; axis = 0: blocks along dimension 0, stored as
 * the cast of the transpose, R = cols and L = rows.  tile = 1: 128 x 128 tiles.
 * Per block, with amax the largest finite |v| and fmax the format's largest number
 * (448, 57344):
 *     factor = min(fmax / amax, 2^126), the Float32 quotient cut to 16
 *              significant bits (toward zero)
 *     scale  = 1 / factor, a Float32 quotient
 *     elem   = the element nearest to the Float32 product v * factor, ties to
 *              even; beyond fmax, fmax; a NaN gives NaN, an infinity NaN (E4M3)
 *              or infinity (E5M2).
 * (The cut makes v * factor exact for bf16 v.  A block of zeros gets scale 2^-126.  It
 * may raise the scale by 2^-15 of itself: a Float32 v that close to the type's largest
 * number can stand for infinity.)
 * Outputs are 16-byte aligned, of the sizes above.
 * MX_ERR_UNSUPPORTED: more than about 2^24 tiles of 128 x 128 (with axis 0 or tile 1;
 * of 128 x 64 with axis 0, tile 0 and bf16), or rows longer than about 2^33 elements (else).
 */
int mx_quantize_b128(const void *src, mx_dtype_t src_dt, int64_t rows, int64_t cols,
                     int64_t ld, int axis, int tile, mx_format_t fmt,
                     void *elems_out, float *scales_out, void *hip_stream);

/* elems * scales, rounded to Float32 and from there to dst_dt, into the row-major
 * dst [rows, cols] with leading dimension ld; arguments as mx_dequantize.  The fill
 * of a partial last block is skipped.  MX_ERR_UNSUPPORTED: as above, with axis 0
 * more than about 2^24 tiles of 128 x 64 whatever the type. */
int mx_dequantize_b128(const void *elems, const float *scales, mx_format_t fmt,
                       int64_t rows, int64_t cols, int axis, int tile,
                       void *dst, mx_dtype_t dst_dt, int64_t ld, void *hip_stream);

/*
 * C[m][n] = sum over blocks b of (sum_{j in b} a[m][j] * b[n][j]) * (sA * sB),
 * A [M][K] and B [N][K] as written by the cast (axis 1, or axis 0 of the transposed
 * source), K a multiple of 128 (else MX_ERR_SHAPE; an odd length is its cast's
 * 128 * ceil(L/128)).  tileA / tileB: 0 = a scale for each row and block,
 * 1 = one for 128 rows and a block.  So for y = x W^T:
 *     forward   A = x (1 x 128),            B = W   (128 x 128)
 *     dx        A = dy (1 x 128),           B = W^T (128 x 128, cast along axis 0)
 *     dW        A = dy^T (1 x 128, axis 0), B = x^T (1 x 128, axis 0)
 * The products of a block go through the matrix instruction, which adds each run of
 * 8 consecutive K products in fixed point with 14 bits below the run's largest
 * product (see mx_gemm); the block's sum is multiplied by the Float32 product of the
 * two scales and added in Float32.  A product of scales has to be inside Float32's
 * range: where it overflows, an entry is infinite or NaN; below 2^-126 it loses bits.
 * The blocks of an entry are added in the order of K, or in the order of K within each
 * half or eighth of K and these sums in order; which, depends on the shape alone:
 * results are reproducible.
 * C, c_dt, ldc, alignment as mx_gemm (scales 16-byte aligned too).  rows of C beyond
 * M and columns beyond N are not touched.
 * MX_ERR_UNSUPPORTED: more than 2^22 tiles of C (of 128 x 128 at least), N of 2^29
 * and more with M up to 32, or K of 2^38 and more.
 */
int mx_gemm_b128(int64_t M, int64_t N, int64_t K,
                 const void *A_elems, const float *A_scales, int tileA, mx_format_t fmtA,
                 const void *B_elems, const float *B_scales, int tileB, mx_format_t fmtB,
                 void *C, mx_dtype_t c_dt, int64_t ldc, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
