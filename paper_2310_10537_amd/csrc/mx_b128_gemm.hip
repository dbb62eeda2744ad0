// Dispatch of the products with a scale per 128 (kernels in mx_b128_gemm.hpp, mx_b128_gemm_few.hpp).
#include "mx_b128_gemm_few.hpp"
#include "mx_b128_gemm_tile.hpp"

namespace mx {

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int WM, int WN>
static hipError_t launch_tiles(const Gemm128 &g, hipStream_t st)
{
    const int64_t tm = (g.M + 16 * MB * WM - 1) / (16 * MB * WM), tn = (g.N + 16 * NB * WN - 1) / (16 * NB * WN);
    if (tm > ((int64_t)1 << 22) / tn) return hipErrorNotSupported;     // (the runtime counts a grid's threads in 32 bits)
    const Bands order = bands(tm, tn, 6);
    hipLaunchKernelGGL((gemm128_kernel<FA, FB, CDT, ROWS_B, MB, NB, WM, WN>), dim3(8 * order.per_xcd), dim3(64 * WM * WN), 0, st, g, order);
    return hipGetLastError();
}

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int AHEAD>
static hipError_t launch_few(const Gemm128 &g, hipStream_t st)
{
    const int64_t gx = (g.N + 16 * NB - 1) / (16 * NB), gy = (g.M + 16 * MB - 1) / (16 * MB);
    if (gx >= (int64_t)1 << 23) return hipErrorNotSupported;           // (the runtime counts a grid's threads in 32 bits; gy is at most 256)
    hipLaunchKernelGGL((gemm128_few_kernel<FA, FB, CDT, ROWS_B, MB, NB, AHEAD>), dim3((unsigned)gx, (unsigned)gy), dim3(512), 0, st, g);
    return hipGetLastError();
}

// Which form.  Measured at K = 4096 with E4M3 operands and 128 x 128 scales of B unless stated (us):
//   up to 16 rows      eight waves share K.  16 columns a work-group: 1 x 4096 5.2, 1 x 11008 11.4, 16 x 11008 16.5; 64 columns: 12.7, 14.1, 15.9.  Wide
//                      matrices (28672, K = 8192) give 64 columns work-groups enough, and read A a quarter as often: 16 rows 72 and 56-62.  The rule looks at N
//                      alone, so at 16 x 11008 it takes the form that is 4 % behind, for the sake of the one row that is 10 % ahead.
//   one round          (up to 256 work-groups) of few-rows kernels with 16 x 16, 32 x 16 or 32 x 32 entries, the smallest that gives one: 128 x 256 6.9 us, 9.6,
//                      11.1, tiles of 128 x 128 16.4; 128 x 1024 11.5 (two rounds), 9.9, 11.9, 16.7; 256 x 1024 20.7 (four), 18.0 (two), 12.0, 16.8; K = 16384,
//                      128 x 256: 21, 31, 40, 65; K = 1024, 512 x 512: 7.3, 6.6, 4.8, 7.7.  Two rounds of 32 x 32 lose: 128 x 4096 23.4, tiles 20.5.
//   up to 32 rows      beyond that, 32 x 64 entries a work-group: 32 x 11008 18.4, tiles 19.6.  With a scale a row of B 27.7: the 32 scales of a block on its way
//                      spill 30 registers (124 bytes a lane).
//   beyond             tiles, of the size whose rounds over the 256 compute units take least: a round of 128 x 128 tiles (K in halves, of as many blocks each) takes about
//                      21, of 256 x 128 34, of 256 x 256 55 (1000 x 4096: 24, 32, 45; 2048 x 4096: 44, 37, 46; 4096 x 4096: 88, 70, 59; 512 x 11008: 42, 33, -).
//   under four blocks  (K up to 384), and K of 2^24 and more, which the tiles' 32-bit offsets do not reach: tiles of four waves.
template <int FA, int FB, int CDT, bool ROWS_B>
static hipError_t launch_rows(const Gemm128 &g, hipStream_t st)
{
    if (g.M <= 16) return g.N < 16384 ? launch_few<FA, FB, CDT, ROWS_B, 1, 1, 4>(g, st) : launch_few<FA, FB, CDT, ROWS_B, 1, 4, 2>(g, st);
    auto count = [](int64_t n, int b) { const int64_t t = (n + b - 1) / b; return t < (int64_t)1 << 30 ? t : (int64_t)1 << 30; };
    auto rounds = [&](int bm, int bn) { return (count(g.M, bm) * count(g.N, bn) + 255) / 256; };
    if (rounds(16, 16) == 1) return launch_few<FA, FB, CDT, ROWS_B, 1, 1, 4>(g, st);
    if (rounds(32, 16) == 1) return launch_few<FA, FB, CDT, ROWS_B, 2, 1, 4>(g, st);
    if (rounds(32, 32) == 1) return launch_few<FA, FB, CDT, ROWS_B, 2, 2, 2>(g, st);
    if (g.M <= 32) return launch_few<FA, FB, CDT, ROWS_B, 2, 4, 2>(g, st);
    const int64_t T = g.K / 128;
    if (T < TILE_MIN_BLOCKS || T >= 1 << 17) return launch_tiles<FA, FB, CDT, ROWS_B, 4, 4, 2, 2>(g, st);
    const int64_t c256 = 55 * rounds(256, 256), c2x1 = 34 * rounds(256, 128), c128 = 21 * rounds(128, 128);
    if (T >= 2 * TILE_MIN_BLOCKS && T % 2 == 0 && c128 < c256 && c128 <= c2x1) return launch_tile<FA, FB, CDT, ROWS_B, 4, 4, 2, 2, 2>(g, st);
    if (c2x1 < c256) return launch_tile<FA, FB, CDT, ROWS_B, 4, 4, 4, 2, 1>(g, st);
    return launch_tile<FA, FB, CDT, ROWS_B, 4, 8, 4, 2, 1>(g, st);
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
