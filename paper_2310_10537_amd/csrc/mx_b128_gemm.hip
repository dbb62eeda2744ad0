// Dispatch of the products with a scale per 128 (kernels in mx_b128_gemm.hpp, mx_b128_gemm_few.hpp).
#include "mx_b128_gemm_few.hpp"
#include "mx_b128_gemm_tile.hpp"

namespace mx {

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int WM, int WN>
static hipError_t launch_tiles(const Gemm128 &g, hipStream_t st)
{
    const int64_t tm = (g.M + 16 * MB * WM - 1) / (16 * MB * WM), tn = (g.N + 16 * NB * WN - 1) / (16 * NB * WN);
    if (tm > ((int64_t)1 << 30) / tn) return hipErrorNotSupported;
    const Bands order = bands(tm, tn, 6);
    hipLaunchKernelGGL((gemm128_kernel<FA, FB, CDT, ROWS_B, MB, NB, WM, WN>), dim3(8 * order.per_xcd), dim3(64 * WM * WN), 0, st, g, order);
    return hipGetLastError();
}

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int AHEAD>
static hipError_t launch_few(const Gemm128 &g, hipStream_t st)
{
    const int64_t gx = (g.N + 16 * NB - 1) / (16 * NB), gy = (g.M + 16 * MB - 1) / (16 * MB);
    if (gx > ((int64_t)1 << 31) - 1 || gy > 65535) return hipErrorNotSupported;
    hipLaunchKernelGGL((gemm128_few_kernel<FA, FB, CDT, ROWS_B, MB, NB, AHEAD>), dim3((unsigned)gx, (unsigned)gy), dim3(512), 0, st, g);
    return hipGetLastError();
}

template <int FA, int FB, int CDT, bool ROWS_B>
static hipError_t launch_rows(const Gemm128 &g, hipStream_t st)
{
    if (g.M <= 16) return launch_few<FA, FB, CDT, ROWS_B, 1, 1, 4>(g, st);
    if (g.M <= 32) return launch_few<FA, FB, CDT, ROWS_B, 2, 1, 2>(g, st);
    if (g.M <= 64) return launch_few<FA, FB, CDT, ROWS_B, 4, 1, 2>(g, st);
    const int64_t large = ((g.M + 255) / 256) * ((g.N + 255) / 256);
    const int64_t T = g.K / 128;
    if (large >= 200 && T >= TILE_MIN_BLOCKS && T < 1 << 17) return launch_tile<FA, FB, CDT, ROWS_B, 4, 8, 4, 2, 1>(g, st);
    if (T >= 2 * TILE_MIN_BLOCKS && T % 2 == 0 && T < 1 << 17) return launch_tile<FA, FB, CDT, ROWS_B, 4, 4, 2, 2, 2>(g, st);
    return launch_tiles<FA, FB, CDT, ROWS_B, 4, 4, 2, 2>(g, st);
}

template <int FA, int FB>
static hipError_t launch_pair(const Gemm128 &g, int c_dt, hipStream_t st)
{
    if (g.b_shift) return c_dt == DT_BF16 ? launch_rows<FA, FB, DT_BF16, false>(g, st) : launch_rows<FA, FB, DT_F32, false>(g, st);
    return c_dt == DT_BF16 ? launch_rows<FA, FB, DT_BF16, true>(g, st) : launch_rows<FA, FB, DT_F32, true>(g, st);
}

hipError_t launch_gemm_b128(int64_t M, int64_t N, int64_t K, const uint8_t *Ae, const float *As, bool tileA, int fmtA, const uint8_t *Be, const float *Bs, bool tileB,
                            int fmtB, void *C, int c_dt, int64_t ldc, hipStream_t st)
{
    const Gemm128 g = {M, N, K, Ae, Be, As, Bs, tileA ? 7 : 0, tileB ? 7 : 0, C, ldc};
    if (K / 128 > ((int64_t)1 << 31) - 16) return hipErrorNotSupported;
    if (fmtA == FP8_E4M3) return fmtB == FP8_E4M3 ? launch_pair<FP8_E4M3, FP8_E4M3>(g, c_dt, st) : launch_pair<FP8_E4M3, FP8_E5M2>(g, c_dt, st);
    return fmtB == FP8_E4M3 ? launch_pair<FP8_E5M2, FP8_E4M3>(g, c_dt, st) : launch_pair<FP8_E5M2, FP8_E5M2>(g, c_dt, st);
}

}  // namespace mx
