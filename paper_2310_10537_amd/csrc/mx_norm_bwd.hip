// Gradients of the RMS norm y = h rstd w (the cast behind it passes its gradient through), with g = dy w and xhat = h rstd:
//     dx = rstd (g - xhat mean(g xhat)) + dh,        dweight = sum over rows of dy xhat.
// dx is the gradient of x and of the residual alike; dh is the gradient that reaches h past the layer.
// Bound by memory: dy, h (and dh) read and dx written, once; everything else is small.  16384 x 2048 bf16 with a dh 49.6 us with dweight (5.4 TB/s), of
// which the lines of partial sums take 4 to 5; 2048 x 16384 63 (4.3 TB/s: two vectors a thread, nothing on its way during a row's sum).
//
// norm_bwd_kernel: a number of work-groups that the shape fixes walks the rows; a row lies in registers, a vector of eight columns a thread
// (two beyond 8192 columns; a wave a row up to 512), the weight is kept from row to row, and every thread adds up its own columns'
// part of dweight in Float32.  Each work-group writes one line of partial sums to scratch memory and
// norm_bwd_weight_kernel adds the lines in a fixed order: no atomics, the same bits every time.
// norm_bwd_long_kernel and norm_bwd_long_weight_kernel: rows that do not fit in registers; dy and h are read three times: 1024 x 32768 with a dh 105 us, 64 x 131072 181.
#include "mx_norm.hpp"

namespace mx {

struct NormBwdArgs {
    const void *dy, *h, *weight, *dh;
    const float *rstd;
    void *dx;
    float *partial;       // [lines][cols], or nullptr: no dweight
    int64_t rows, cols, lddy, ldh, lddh, lddx;
    int w_dt;
    int64_t row0;         // (norm_bwd_long_kernel) first row of a launch
};

template <int DT> struct Vec8 { uint32_t d[DT == DT_BF16 ? 4 : 8]; };

// eight elements as they lie in memory (n of them; the rest zero), and one of them as Float32
template <int DT>
__device__ __forceinline__ Vec8<DT> fetch8(const void *p, int64_t at, int n)
{
    Vec8<DT> v;
    if constexpr (DT == DT_BF16) {
        const uint16_t *q = static_cast<const uint16_t *>(p) + at;
        if (n >= 8) {
            const uint4 t = ld16_nt(q);
            v.d[0] = t.x; v.d[1] = t.y; v.d[2] = t.z; v.d[3] = t.w;
        } else {
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; i++) e[i] = i < n ? q[i] : 0u;
#pragma unroll
            for (int i = 0; i < 4; i++) v.d[i] = e[2 * i] | (e[2 * i + 1] << 16);
        }
    } else {
        const uint32_t *q = static_cast<const uint32_t *>(p) + at;
        if (n >= 8) {
            const uint4 a = ld16_nt(q), b = ld16_nt(q + 4);
            v.d[0] = a.x; v.d[1] = a.y; v.d[2] = a.z; v.d[3] = a.w;
            v.d[4] = b.x; v.d[5] = b.y; v.d[6] = b.z; v.d[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v.d[i] = i < n ? q[i] : 0u;
        }
    }
    return v;
}
template <int DT>
__device__ __forceinline__ float elem(const Vec8<DT> &v, int i)
{
    if constexpr (DT == DT_BF16) return __uint_as_float(i & 1 ? v.d[i >> 1] & 0xFFFF0000u : v.d[i >> 1] << 16);
    else return __uint_as_float(v.d[i]);
}

__device__ __forceinline__ void load_weight(const NormBwdArgs &a, int64_t col, int n, float (&w)[8])
{
    if (!a.weight) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = 1.0f;
    } else if (a.w_dt == DT_BF16) {
        load8<DT_BF16, false>(a.weight, col, n, w);
    } else {
        load8<DT_F32, false>(a.weight, col, n, w);
    }
}

template <int DT, int VPT, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_bwd_kernel(NormBwdArgs a)
{
    __shared__ float lds[WAVE ? 256 * 8 : 2 * 16];
    const int nt = WAVE ? 64 : (int)blockDim.x, t = WAVE ? threadIdx.x & 63 : threadIdx.x;
    constexpr int RPW = WAVE ? 4 : 1;                 // rows a work-group has in hand
    float w[VPT][8], dw[VPT][8];
#pragma unroll
    for (int k = 0; k < VPT; k++) {
        const int64_t col = (int64_t)(k * nt + t) * 8;
        load_weight(a, col, inside(a.cols - col, 8), w[k]);
#pragma unroll
        for (int i = 0; i < 8; i++) dw[k][i] = 0.0f;
    }
    const float inv = 1.0f / (float)a.cols;
    const int64_t first = (int64_t)blockIdx.x * RPW + (WAVE ? threadIdx.x >> 6 : 0), pitch = (int64_t)gridDim.x * RPW;
    // a row's vectors and its rstd, requested one row ahead: the sum over a row, and the barrier in it, would leave the memory idle (4096 x
    // 8192 bf16 58 us without, 51 with).  Two vectors a thread leave no registers for that in a work-group of 1024.
    constexpr bool AHEAD = VPT == 1;
    Vec8<DT> dy1[VPT], h1[VPT], dh1[VPT];
    float rstd1 = 0.0f;
    auto request = [&](int64_t row) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < VPT; k++) {
            const int64_t col = (int64_t)(k * nt + t) * 8;
            const int n = inside(a.cols - col, 8);
            dy1[k] = fetch8<DT>(a.dy, row * a.lddy + col, n);
            h1[k] = fetch8<DT>(a.h, row * a.ldh + col, n);
            if (a.dh) dh1[k] = fetch8<DT>(a.dh, row * a.lddh + col, n);
        }
        rstd1 = a.rstd[row];
    };
    if (AHEAD && first < a.rows) request(first);
    int trip = 0;
    for (int64_t row = first; row < a.rows; row += pitch, trip ^= 1) {
        if (!AHEAD) request(row);
        Vec8<DT> dy[VPT], h[VPT], dh[VPT];
#pragma unroll
        for (int k = 0; k < VPT; k++) { dy[k] = dy1[k]; h[k] = h1[k]; dh[k] = dh1[k]; }
        const float rstd = rstd1;
        if (AHEAD && row + pitch < a.rows) request(row + pitch);
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < VPT; k++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float d = elem<DT>(dy[k], i), x = elem<DT>(h[k], i) * rstd;
                sum = fmaf(d * w[k][i], x, sum);
                dw[k][i] = fmaf(d, x, dw[k][i]);
            }
        // (two places in LDS taken in turn: the barrier in between keeps a fast wave from writing where a slow one still reads)
        const float mean = row_sum<WAVE>(sum, lds + (WAVE ? 0 : trip * 16)) * inv;
#pragma unroll
        for (int k = 0; k < VPT; k++) {
            const int64_t col = (int64_t)(k * nt + t) * 8;
            const int n = inside(a.cols - col, 8);
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float g = elem<DT>(dy[k], i) * w[k][i], x = elem<DT>(h[k], i) * rstd;
                dx[i] = rstd * fmaf(-x, mean, g);
            }
            if (a.dh) {
#pragma unroll
                for (int i = 0; i < 8; i++) dx[i] += elem<DT>(dh[k], i);
            }
            if (n > 0) put8<DT>(a.dx, row * a.lddx + col, n, dx);
        }
    }
    if (!a.partial) return;
    float *line = a.partial + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int k = 0; k < VPT; k++) {
        const int64_t col = (int64_t)(k * nt + t) * 8;
        const int n = inside(a.cols - col, 8);
        if constexpr (WAVE) {                         // four rows at a time: their waves' sums in pairs
#pragma unroll
            for (int i = 0; i < 8; i++) lds[threadIdx.x * 8 + i] = dw[k][i];
            __syncthreads();
            if (threadIdx.x < 64) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float v = (lds[t * 8 + i] + lds[(64 + t) * 8 + i]) + (lds[(128 + t) * 8 + i] + lds[(192 + t) * 8 + i]);
                    if (i < n) line[col + i] = v;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) line[col + i] = dw[k][i];
        }
    }
}

// dweight[c] = partial[0][c] + partial[1][c] + ..., 16 columns and 64 runs of lines (every 64th) a work-group
__global__ __launch_bounds__(1024) void norm_bwd_weight_kernel(const float *__restrict__ partial, int lines, int64_t pitch, int64_t cols, float *__restrict__ dweight)
{
    __shared__ float part[64][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;
    // eight lines of a run at a time, and then the 64 runs, joined in pairs, and these in pairs: eleven roundings at most up to 1024 lines
    // (333 x 1000 Float32, Gaussian: dweight's error 1.7e-7 of it and 8.1 us for both kernels with everything one after the other, 8.8e-8 and 7.0 so)
    float sum = 0.0f;
    if (col < cols) {
        for (int l = g; l < lines; l += 512) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = l + 64 * j < lines ? partial[(int64_t)(l + 64 * j) * pitch + col] : 0.0f;
            sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
    }
    part[g][c] = sum;
#pragma unroll
    for (int n = 16; n > 0; n >>= 2) {
        __syncthreads();
        if (g < n) part[g][c] = (part[g][c] + part[g + n][c]) + (part[g + 2 * n][c] + part[g + 3 * n][c]);
    }
    if (g == 0 && col < cols) dweight[col] = part[0][c];
}

template <int DT>
__global__ __launch_bounds__(256) void norm_bwd_long_kernel(NormBwdArgs a)
{
    __shared__ float lds[4];
    const int64_t row = a.row0 + blockIdx.x;
    const float rstd = a.rstd[row];
    float sum = 0.0f;
    for (int64_t col = threadIdx.x * 8; col < a.cols; col += 2048) {
        const int n = inside(a.cols - col, 8);
        float w[8];
        load_weight(a, col, n, w);
        const Vec8<DT> dy = fetch8<DT>(a.dy, row * a.lddy + col, n), h = fetch8<DT>(a.h, row * a.ldh + col, n);
#pragma unroll
        for (int i = 0; i < 8; i++) sum = fmaf(elem<DT>(dy, i) * w[i], elem<DT>(h, i) * rstd, sum);
    }
    const float mean = row_sum<false>(sum, lds) / (float)a.cols;
    for (int64_t col = threadIdx.x * 8; col < a.cols; col += 2048) {
        const int n = inside(a.cols - col, 8);
        float w[8], dx[8];
        load_weight(a, col, n, w);
        const Vec8<DT> dy = fetch8<DT>(a.dy, row * a.lddy + col, n), h = fetch8<DT>(a.h, row * a.ldh + col, n);
#pragma unroll
        for (int i = 0; i < 8; i++) dx[i] = rstd * fmaf(-elem<DT>(h, i) * rstd, mean, elem<DT>(dy, i) * w[i]);
        if (a.dh) {
            const Vec8<DT> dh = fetch8<DT>(a.dh, row * a.lddh + col, n);
#pragma unroll
            for (int i = 0; i < 8; i++) dx[i] += elem<DT>(dh, i);
        }
        put8<DT>(a.dx, row * a.lddx + col, n, dx);
    }
}

// partial sums of dweight over the rows of line blockIdx.y, 2048 columns a work-group
template <int DT>
__global__ __launch_bounds__(256) void norm_bwd_long_weight_kernel(NormBwdArgs a)
{
    const int64_t col = (int64_t)blockIdx.x * 2048 + threadIdx.x * 8;
    const int n = inside(a.cols - col, 8);
    if (n == 0) return;
    float dw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row];
        const Vec8<DT> dy = fetch8<DT>(a.dy, row * a.lddy + col, n), h = fetch8<DT>(a.h, row * a.ldh + col, n);
#pragma unroll
        for (int i = 0; i < 8; i++) dw[i] = fmaf(elem<DT>(dy, i), elem<DT>(h, i) * rstd, dw[i]);
    }
    float *line = a.partial + (int64_t)blockIdx.y * a.cols;
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) line[col + i] = dw[i];
}

// Columns that fit in registers, and threads of a work-group for so many
constexpr int64_t NORM_BWD_COLS = 16384;
static int norm_bwd_threads(int64_t cols)
{
    const int64_t nvec = (cols + 7) / 8;
    return nvec <= 64 ? 256 : nvec <= 1024 ? (int)((nvec + 63) / 64 * 64) : (int)((nvec + 127) / 128 * 64);
}

// Lines of partial sums: as many work-groups as give each compute unit 512 threads, one at least, fewer where there are fewer rows.  (16384 x 2048
// bf16 50.5 us so, 53.7 with 1024 threads, 60 with 2048; 8192 x 4096 49.7, 51.4, 58.)
int norm_bwd_lines(int64_t rows, int64_t cols)
{
    if (cols > NORM_BWD_COLS) return (int)(rows < 64 ? rows : 64);
    const int64_t need = cols <= 512 ? (rows + 3) / 4 : rows, threads = norm_bwd_threads(cols), most = threads < 512 ? 256 * (512 / threads) : 256;
    return (int)(need < most ? need : most);
}

size_t norm_bwd_workspace(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0) return 0;
    return ((size_t)norm_bwd_lines(rows, cols) * (size_t)cols * 4 + 255) & ~(size_t)255;
}

static void launch_norm_bwd_weight(const float *partial, int lines, int64_t cols, float *dweight, hipStream_t st)
{
    constexpr int64_t MOST = (int64_t)1 << 25;        // columns a launch: the runtime counts a grid's threads in 32 bits
    for (int64_t c0 = 0; c0 < cols; c0 += MOST) {
        const int64_t n = cols - c0 < MOST ? cols - c0 : MOST;
        hipLaunchKernelGGL(norm_bwd_weight_kernel, dim3((unsigned)((n + 15) / 16)), dim3(1024), 0, st, partial ? partial + c0 : nullptr, lines, cols, n, dweight + c0);
    }
}

template <int DT>
static hipError_t launch_norm_bwd_t(const NormBwdArgs &a, int lines, float *dweight, hipStream_t st)
{
    const dim3 b(256), g((unsigned)lines);
    if (a.cols > NORM_BWD_COLS) {
        if (a.partial)                                // first: dx may take the place of dy
            hipLaunchKernelGGL((norm_bwd_long_weight_kernel<DT>), dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)lines), b, 0, st, a);
        const int64_t most = rows_per_launch(256);
        for (int64_t r0 = 0; r0 < a.rows; r0 += most) {
            NormBwdArgs part = a;
            part.row0 = r0;
            hipLaunchKernelGGL((norm_bwd_long_kernel<DT>), dim3((unsigned)(a.rows - r0 < most ? a.rows - r0 : most)), b, 0, st, part);
        }
    } else {
        const dim3 threads(norm_bwd_threads(a.cols));
        if (a.cols <= 512) hipLaunchKernelGGL((norm_bwd_kernel<DT, 1, true>), g, threads, 0, st, a);
        else if (a.cols <= 8192) hipLaunchKernelGGL((norm_bwd_kernel<DT, 1, false>), g, threads, 0, st, a);
        else hipLaunchKernelGGL((norm_bwd_kernel<DT, 2, false>), g, threads, 0, st, a);
    }
    if (a.partial) launch_norm_bwd_weight(a.partial, lines, a.cols, dweight, st);
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *weight, int w_dt, const float *rstd, const void *dh, int64_t lddh,
                           int dt, int64_t rows, int64_t cols, void *dx, int64_t lddx, float *dweight, hipStream_t st)
{
    NormBwdArgs a = {dy, h, weight, dh, rstd, dx, nullptr, rows, cols, lddy, ldh, lddh, lddx, w_dt, 0};
    if (rows == 0) {                                  // an empty sum
        launch_norm_bwd_weight(nullptr, 0, cols, dweight, st);
        return hipGetLastError();
    }
    uint8_t *ws = nullptr;
    if (dweight) {
        const hipError_t e = ws_acquire(norm_bwd_workspace(rows, cols), st, &ws);
        if (e != hipSuccess) return e;
        a.partial = reinterpret_cast<float *>(ws);
    }
    const int lines = norm_bwd_lines(rows, cols);
    hipError_t e = dt == DT_BF16 ? launch_norm_bwd_t<DT_BF16>(a, lines, dweight, st) : launch_norm_bwd_t<DT_F32>(a, lines, dweight, st);
    if (ws) {
        const hipError_t r = ws_release(ws, st);
        if (e == hipSuccess) e = r;
    }
    return e;
}

}  // namespace mx
