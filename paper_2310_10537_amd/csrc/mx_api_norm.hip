// C ABI of the 128-element scaling and of the RMS norm (include/mx_b128.h, include/mx_norm.h): argument
// validation and dispatch, as in mx_api.hip.
#include "../../include/mx_norm.h"

#include "mx_norm.hpp"

namespace {

bool fmt8_ok(int f) { return f == MX_FP8_E4M3 || f == MX_FP8_E5M2; }
bool dt_ok(int d) { return d == MX_DT_F32 || d == MX_DT_BF16; }
bool flag_ok(int v) { return v == 0 || v == 1; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t esize(int dt) { return dt == MX_DT_BF16 ? 2 : 4; }
int64_t up128(int64_t n) { return (n + 127) / 128; }
int status(hipError_t e)
{
    return e == hipSuccess ? MX_OK : e == hipErrorNotSupported ? MX_ERR_UNSUPPORTED : e == hipErrorOutOfMemory ? MX_ERR_WORKSPACE : MX_ERR_LAUNCH;
}
constexpr int64_t MAX_LEN = (int64_t)1 << 62;         // sizes whose rounded-up form still fits

// one tensor of rows: present ones need alignment and a pitch
bool rows_aligned(const void *p, int64_t ld, int dt) { return !p || (aligned16(p) && (ld * esize(dt)) % 16 == 0); }
bool pitch_ok(const void *p, int64_t ld, int64_t cols) { return !p || (ld >= cols && ld <= MAX_LEN / 8); }

int rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, int w_dt, int dt, int64_t rows, int64_t cols, float eps, int out, int rnd,
            void *elems, void *scales, void *h, int64_t ldh, void *y, int64_t ldy, float *rstd, void *hip_stream)
{
    if (!dt_ok(dt) || (weight && !dt_ok(w_dt)) || !(eps >= 0.0f && eps <= 3.4028234e38f)) return MX_ERR_ENUM;
    if (rows < 0 || cols < 0 || cols > MAX_LEN || ldx < cols || !pitch_ok(residual, ldr, cols) || !pitch_ok(h, ldh, cols) || !pitch_ok(y, ldy, cols)) return MX_ERR_SHAPE;
    if (rows == 0 || cols == 0) return MX_OK;
    if (!x || (out == mx::OUT_NONE ? !y : !elems || !scales)) return MX_ERR_NULL;
    if (!rows_aligned(x, ldx, dt) || !rows_aligned(residual, ldr, dt) || !rows_aligned(h, ldh, dt) || !rows_aligned(y, ldy, dt) || !aligned16(weight) ||
        !aligned16(elems) || !aligned16(scales) || (reinterpret_cast<uintptr_t>(rstd) & 3))
        return MX_ERR_ALIGN;
    const int64_t block = mx::out_block(out);
    if (rows >= (int64_t)1 << 31 || cols >= (int64_t)1 << 32) return MX_ERR_UNSUPPORTED;
    const mx::NormArgs a = {x, residual, weight, h, y, static_cast<uint8_t *>(elems), scales, rstd, rows, cols, ldx, ldr, ldh, ldy, eps,
                            w_dt, rnd, (int)((cols + block - 1) / block * (block / 8)), 0};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return status(dt == MX_DT_BF16 ? mx::launch_norm_bf16(a, out, st) : mx::launch_norm_f32(a, out, st));
}

}  // namespace

extern "C" {

size_t mx_b128_elem_bytes(int64_t rows, int64_t cols, int axis)
{
    if (rows < 0 || cols < 0 || rows > MAX_LEN || cols > MAX_LEN || !flag_ok(axis)) return 0;
    const int64_t lines = axis == 1 ? rows : cols, len = axis == 1 ? cols : rows;
    return (size_t)lines * (size_t)up128(len) * 128;
}

size_t mx_b128_scale_count(int64_t rows, int64_t cols, int axis, int tile)
{
    if (rows < 0 || cols < 0 || rows > MAX_LEN || cols > MAX_LEN || !flag_ok(axis) || !flag_ok(tile)) return 0;
    const int64_t lines = axis == 1 ? rows : cols, len = axis == 1 ? cols : rows;
    return (size_t)(tile ? up128(lines) : lines) * (size_t)up128(len);
}

int mx_quantize_b128(const void *src, mx_dtype_t src_dt, int64_t rows, int64_t cols, int64_t ld, int axis, int tile, mx_format_t fmt, void *elems_out, float *scales_out,
                     void *hip_stream)
{
    if (!fmt8_ok(fmt) || !dt_ok(src_dt) || !flag_ok(axis) || !flag_ok(tile)) return MX_ERR_ENUM;
    if (rows < 0 || cols < 0 || rows > MAX_LEN || cols > MAX_LEN || ld < cols) return MX_ERR_SHAPE;
    if (rows == 0 || cols == 0) return MX_OK;
    if (!src || !elems_out || !scales_out) return MX_ERR_NULL;
    if (!aligned16(src) || !aligned16(elems_out) || !aligned16(scales_out) || (ld * esize(src_dt)) % 16) return MX_ERR_ALIGN;
    return status(mx::launch_cast_b128(src, src_dt, rows, cols, ld, axis, tile != 0, fmt, static_cast<uint8_t *>(elems_out), scales_out, static_cast<hipStream_t>(hip_stream)));
}

int mx_dequantize_b128(const void *elems, const float *scales, mx_format_t fmt, int64_t rows, int64_t cols, int axis, int tile, void *dst, mx_dtype_t dst_dt, int64_t ld,
                       void *hip_stream)
{
    if (!fmt8_ok(fmt) || !dt_ok(dst_dt) || !flag_ok(axis) || !flag_ok(tile)) return MX_ERR_ENUM;
    if (rows < 0 || cols < 0 || rows > MAX_LEN || cols > MAX_LEN || ld < cols) return MX_ERR_SHAPE;
    if (rows == 0 || cols == 0) return MX_OK;
    if (!elems || !scales || !dst) return MX_ERR_NULL;
    if (!aligned16(elems) || !aligned16(scales) || !aligned16(dst) || (ld * esize(dst_dt)) % 16) return MX_ERR_ALIGN;
    return status(mx::launch_dequant_b128(static_cast<const uint8_t *>(elems), scales, fmt, rows, cols, axis, tile != 0, dst, dst_dt, ld, static_cast<hipStream_t>(hip_stream)));
}

int mx_gemm_b128(int64_t M, int64_t N, int64_t K, const void *A_elems, const float *A_scales, int tileA, mx_format_t fmtA, const void *B_elems, const float *B_scales,
                 int tileB, mx_format_t fmtB, void *C, mx_dtype_t c_dt, int64_t ldc, void *hip_stream)
{
    if (!fmt8_ok(fmtA) || !fmt8_ok(fmtB) || !dt_ok(c_dt) || !flag_ok(tileA) || !flag_ok(tileB)) return MX_ERR_ENUM;
    if (M < 0 || N < 0 || K < 0 || K % 128 || M > MAX_LEN || N > MAX_LEN || ldc < N) return MX_ERR_SHAPE;
    if (M == 0 || N == 0) return MX_OK;
    if (!C || (K > 0 && (!A_elems || !A_scales || !B_elems || !B_scales))) return MX_ERR_NULL;
    if (!aligned16(A_elems) || !aligned16(A_scales) || !aligned16(B_elems) || !aligned16(B_scales) || !aligned16(C)) return MX_ERR_ALIGN;
    return status(mx::launch_gemm_b128(M, N, K, static_cast<const uint8_t *>(A_elems), A_scales, tileA != 0, fmtA, static_cast<const uint8_t *>(B_elems), B_scales,
                                       tileB != 0, fmtB, C, c_dt, ldc, static_cast<hipStream_t>(hip_stream)));
}

int mx_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, mx_dtype_t w_dt, mx_dtype_t dt, int64_t rows, int64_t cols, float eps,
               void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out, void *hip_stream)
{
    return rmsnorm(x, ldx, residual, ldr, weight, w_dt, dt, rows, cols, eps, mx::OUT_NONE, 0, nullptr, nullptr, h_out, ldh, y_out, ldy, rstd_out, hip_stream);
}

int mx_rmsnorm_q(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, mx_dtype_t w_dt, mx_dtype_t dt, int64_t rows, int64_t cols, float eps,
                 mx_format_t fmt, mx_round_t rnd, void *elems_out, uint8_t *scales_out, void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out,
                 void *hip_stream)
{
    if ((int)fmt < 0 || (int)fmt >= mx::NUM_FORMATS || (int)rnd < 0 || (int)rnd > MX_ROUND_TOWARD_ZERO) return MX_ERR_ENUM;
    return rmsnorm(x, ldx, residual, ldr, weight, w_dt, dt, rows, cols, eps, fmt, rnd, elems_out, scales_out, h_out, ldh, y_out, ldy, rstd_out, hip_stream);
}

int mx_rmsnorm_b128(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, mx_dtype_t w_dt, mx_dtype_t dt, int64_t rows, int64_t cols, float eps,
                    mx_format_t fmt, void *elems_out, float *scales_out, void *h_out, int64_t ldh, void *y_out, int64_t ldy, float *rstd_out, void *hip_stream)
{
    if (!fmt8_ok(fmt)) return MX_ERR_ENUM;
    const int out = fmt == MX_FP8_E4M3 ? mx::OUT_B128_E4M3 : mx::OUT_B128_E5M2;
    return rmsnorm(x, ldx, residual, ldr, weight, w_dt, dt, rows, cols, eps, out, 0, elems_out, scales_out, h_out, ldh, y_out, ldy, rstd_out, hip_stream);
}

size_t mx_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t cols) { return cols > MAX_LEN ? 0 : mx::norm_bwd_workspace(rows, cols); }

int mx_rmsnorm_bwd_ws(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *weight, mx_dtype_t w_dt, const float *rstd, const void *dh, int64_t lddh,
                      mx_dtype_t dt, int64_t rows, int64_t cols, void *dx, int64_t lddx, float *dweight, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!dt_ok(dt) || (weight && !dt_ok(w_dt))) return MX_ERR_ENUM;
    if (rows < 0 || cols < 0 || cols > MAX_LEN || lddy < cols || ldh < cols || lddx < cols || !pitch_ok(dh, lddh, cols)) return MX_ERR_SHAPE;
    if (cols == 0 || (rows == 0 && !dweight)) return MX_OK;
    if (rows > 0 && (!dy || !h || !rstd || !dx)) return MX_ERR_NULL;
    if (!rows_aligned(dy, lddy, dt) || !rows_aligned(h, ldh, dt) || !rows_aligned(dh, lddh, dt) || !rows_aligned(dx, lddx, dt) || !aligned16(weight) || !aligned16(dweight) ||
        (reinterpret_cast<uintptr_t>(rstd) & 3))
        return MX_ERR_ALIGN;
    if (rows >= (int64_t)1 << 31 || cols >= (int64_t)1 << 32) return MX_ERR_UNSUPPORTED;
    if (workspace) {
        if (!aligned16(workspace)) return MX_ERR_ALIGN;
        if (dweight && workspace_bytes < mx::norm_bwd_workspace(rows, cols)) return MX_ERR_WORKSPACE;
    }
    mx::WorkspaceScope scope(workspace, workspace_bytes);
    return status(mx::launch_norm_bwd(dy, lddy, h, ldh, weight, w_dt, rstd, dh, lddh, dt, rows, cols, dx, lddx, dweight, static_cast<hipStream_t>(hip_stream)));
}

int mx_rmsnorm_bwd(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *weight, mx_dtype_t w_dt, const float *rstd, const void *dh, int64_t lddh,
                   mx_dtype_t dt, int64_t rows, int64_t cols, void *dx, int64_t lddx, float *dweight, void *hip_stream)
{
    return mx_rmsnorm_bwd_ws(dy, lddy, h, ldh, weight, w_dt, rstd, dh, lddh, dt, rows, cols, dx, lddx, dweight, nullptr, 0, hip_stream);
}

}  // extern "C"
