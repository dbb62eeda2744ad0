// RMS norm with the residual's addition and a cast of the result:
//     h = x + residual rounded to the tensors' type,  rstd = 1 / sqrt(mean(h^2) + eps),  y = (h w) rstd,
// delivered as any of: h, y in the tensors' type, rstd, and the cast of the Float32 y to an MX format or to 8 bits with a
// Float32 scale per 128.  (h w first: for bf16 h and w that product is exact, so y carries one rounding and that of rstd.)
// Bound by memory: x and the residual read, h and the codes written, all once.  8192 x 4096 bf16 with a residual: 45.1 us with a Float32 scale per 128
// (5.2 TB/s), MX E4M3 42.7-44.9, E2M1 39.8, E3M2 54-56 (its converts want a whole block in a lane, so the exact encoder packs it); one row of 4096 2.8.
//
// norm_kernel: a row stays in registers between the sum of squares and the output: a vector of eight elements a thread and as many threads as
// that takes, two vectors beyond 8192 columns, and for up to 512 columns a wave a row, four rows a work-group.  More vectors a thread and
// fewer threads are slower throughout: 8192 x 4096 bf16 with a residual 44 us with one (512 threads), 45 with two, 48 with four, 58 with eight
// (a wave a row); one row of 4096 3.0, 3.9, 5.6 and 8.9; 2048 x 16384 46 with two vectors, 48 with four, 57 with eight.
// norm_long_kernel: rows beyond 16384 columns; h is read (or added up) a second time.  1024 x 32768 bf16 with a residual 53 us (4.4 TB/s of what has to be
// moved), 64 x 131072 42: a work-group a row leaves most compute units without one.
#pragma once

#include "mx_norm.hpp"

namespace mx {

template <int OUT>
__device__ __forceinline__ void norm_modes()
{
    if constexpr (OUT == FP8_E4M3 || OUT == FP8_E5M2 || OUT == OUT_B128_E4M3 || OUT == OUT_B128_E5M2) fp8_saturate_mode();
}

template <int DT>
__device__ __forceinline__ void load_sum(const NormArgs &a, int64_t row, int64_t col, int n, float (&h)[8])
{
    load8<DT>(a.x, row * a.ldx + col, n, h);
    if (a.residual) {
        float r[8];
        load8<DT>(a.residual, row * a.ldr + col, n, r);
#pragma unroll
        for (int i = 0; i < 8; i++) h[i] = held<DT>(h[i] + r[i]);
    }
}

template <int OUT, int DT>
__device__ __forceinline__ void put_vector(const NormArgs &a, int64_t row, int vec, bool on, const float (&h)[8], float rstd)
{
    const int64_t col = (int64_t)vec * 8;
    const int n = on ? inside(a.cols - col, 8) : 0;
    float y[8], w[8];
    if (a.weight) {
        if (a.w_dt == DT_BF16) load8<DT_BF16, false>(a.weight, col, n, w);
        else load8<DT_F32, false>(a.weight, col, n, w);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) y[i] = i < n ? (a.weight ? h[i] * w[i] : h[i]) * rstd : 0.0f;    // (a NaN or infinite rstd stays out of the fill)
    if (a.y && n > 0) put8<DT>(a.y, row * a.ldy + col, n, y);
    put_cast<OUT>(y, a.rnd, a.elems, a.scales, row, vec, a.nvec, on);
}

template <int OUT, int DT, int VPT, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_kernel(NormArgs a)
{
    norm_modes<OUT>();
    __shared__ float lds[16];
    const int nt = WAVE ? 64 : (int)blockDim.x, t = WAVE ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = a.row0 + (WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x);
    if (WAVE && row >= a.rows) return;                // (a whole wave; the kernel has no barrier then)
    float h[VPT][8], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < VPT; k++) {
        const int64_t col = (int64_t)(k * nt + t) * 8;
        load_sum<DT>(a, row, col, inside(a.cols - col, 8), h[k]);
    }
#pragma unroll
    for (int k = 0; k < VPT; k++) {
        const int64_t col = (int64_t)(k * nt + t) * 8;
        const int n = inside(a.cols - col, 8);
        if (a.h && n > 0) put8<DT>(a.h, row * a.ldh + col, n, h[k]);
#pragma unroll
        for (int i = 0; i < 8; i++) sum = fmaf(h[k][i], h[k][i], sum);
    }
    const float rstd = rsqrtf(row_sum<WAVE>(sum, lds) / (float)a.cols + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < VPT; k++) put_vector<OUT, DT>(a, row, k * nt + t, k * nt + t < a.nvec, h[k], rstd);
}

template <int OUT, int DT>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a)
{
    norm_modes<OUT>();
    __shared__ float lds[16];
    const int64_t row = a.row0 + blockIdx.x;
    float sum = 0.0f;
    for (int vec = threadIdx.x; vec < a.nvec; vec += 1024) {
        const int64_t col = (int64_t)vec * 8;
        const int n = inside(a.cols - col, 8);
        float h[8];
        load_sum<DT>(a, row, col, n, h);
        if (a.h && n > 0) put8<DT>(a.h, row * a.ldh + col, n, h);
#pragma unroll
        for (int i = 0; i < 8; i++) sum = fmaf(h[i], h[i], sum);
    }
    const float rstd = rsqrtf(row_sum<false>(sum, lds) / (float)a.cols + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    const int trips = (a.nvec + 1023) / 1024;           // (the same number for every lane: they share blocks)
    for (int k = 0; k < trips; k++) {
        const int vec = k * 1024 + threadIdx.x;
        const bool on = vec < a.nvec;
        const int64_t col = (int64_t)vec * 8;
        const int n = on ? inside(a.cols - col, 8) : 0;
        float h[8];
        // h may have been written over x or the residual: then it is read where it was written (by this very thread)
        if (a.h) load8<DT, false>(a.h, row * a.ldh + col, n, h);
        else load_sum<DT>(a, row, col, n, h);
        put_vector<OUT, DT>(a, row, vec, on, h, rstd);
    }
}

template <int OUT, int DT>
static hipError_t launch_norm_t(const NormArgs &a, hipStream_t st)
{
    const int threads = a.nvec <= 1024 ? (a.nvec + 63) / 64 * 64 : a.nvec <= 2048 ? (a.nvec + 127) / 128 * 64 : 1024;
    const bool waves = a.nvec <= 64;                  // four rows a work-group of 256
    const int64_t most = rows_per_launch(threads);
    for (int64_t r0 = 0; r0 < a.rows; r0 += most) {
        NormArgs b = a;
        b.row0 = r0;
        const int64_t n = a.rows - r0 < most ? a.rows - r0 : most;
        const dim3 grid((unsigned)(waves ? (n + 3) / 4 : n));
        if (waves) hipLaunchKernelGGL((norm_kernel<OUT, DT, 1, true>), grid, dim3(256), 0, st, b);
        else if (a.nvec <= 1024) hipLaunchKernelGGL((norm_kernel<OUT, DT, 1, false>), grid, dim3(threads), 0, st, b);
        else if (a.nvec <= 2048) hipLaunchKernelGGL((norm_kernel<OUT, DT, 2, false>), grid, dim3(threads), 0, st, b);
        else hipLaunchKernelGGL((norm_long_kernel<OUT, DT>), grid, dim3(threads), 0, st, b);
    }
    return hipGetLastError();
}

}  // namespace mx
