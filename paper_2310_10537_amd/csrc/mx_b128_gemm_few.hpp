// The product of mx_b128_gemm.hpp for few rows of A, where reading B is all that costs: each byte of B is wanted once, so it goes
// straight to registers.  A work-group has 16 NB columns; its eight waves take an eighth of the blocks along K each, load their
// fragments (a lane 32 consecutive bytes of its column) several blocks ahead, and their partial sums are added in a fixed order through LDS.
#pragma once

#include "mx_b128_gemm.hpp"

namespace mx {

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int AHEAD>
__global__ __launch_bounds__(512) void gemm128_few_kernel(Gemm128 g)
{
    constexpr int NW = 8;
    __shared__ __attribute__((aligned(16))) float red[NW - 1][MB * NB][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NB), m0 = (int64_t)blockIdx.y * (16 * MB);
    const int T = (int)(g.K / 128);
    // blocks of this wave: an eighth each, the first T % 8 waves one more
    const int base = T / NW, extra = T % NW;
    const int t0 = wave * base + (wave < extra ? wave : extra), t1 = t0 + base + (wave < extra ? 1 : 0);

    const uint8_t *pA[MB], *pB[NB];
    const float *sA[MB], *sB[NB];
#pragma unroll
    for (int x = 0; x < MB; x++) {
        const int64_t row = m0 + 16 * x + i < g.M ? m0 + 16 * x + i : g.M - 1;
        pA[x] = g.Ae + row * g.K + 32 * q;
        sA[x] = g.As + (row >> g.a_shift) * T;
    }
#pragma unroll
    for (int y = 0; y < NB; y++) {
        const int64_t row = n0 + 16 * y + i < g.N ? n0 + 16 * y + i : g.N - 1;
        pB[y] = g.Be + row * g.K + 32 * q;
        // ROWS_B: the scales of the lane's four columns are consecutive rows (clamped one by one below)
        sB[y] = g.Bs + (ROWS_B ? 0 : ((n0 + 16 * y < g.N ? n0 + 16 * y : g.N - 1) >> 7) * T);
    }
    v4f_t acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) acc[x][y] = v4f_t{0.f, 0.f, 0.f, 0.f};

    auto load = [](const uint8_t *p) {
        const uint4 lo = ld16(p), hi = ld16(p + 16);
        return v8i_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };
    auto load_nt = [](const uint8_t *p) {
        const uint4 lo = ld16_nt(p), hi = ld16_nt(p + 16);
        return v8i_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };
    for (int t = t0; t < t1; t += AHEAD) {
        v8i_t a[AHEAD][MB], b[AHEAD][NB];
        float sa[AHEAD][MB], sb[AHEAD][NB][ROWS_B ? 4 : 1];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int tt = t + u < t1 ? t + u : t1 - 1;              // (a block beyond the range: the last one again, scaled by zero)
#pragma unroll
            for (int y = 0; y < NB; y++) b[u][y] = g.M <= 16 * MB ? load_nt(pB[y] + (int64_t)tt * 128) : load(pB[y] + (int64_t)tt * 128);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int tt = t + u < t1 ? t + u : t1 - 1;
#pragma unroll
            for (int x = 0; x < MB; x++) {
                a[u][x] = load(pA[x] + (int64_t)tt * 128);
                sa[u][x] = sA[x][tt];
            }
#pragma unroll
            for (int y = 0; y < NB; y++) {
                if constexpr (ROWS_B) {
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int64_t c = n0 + 16 * y + 4 * q + e;
                        sb[u][y][e] = g.Bs[(c < g.N ? c : g.N - 1) * T + tt];
                    }
                } else {
                    sb[u][y][0] = sB[y][tt];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (t + u >= t1) break;
#pragma unroll
            for (int x = 0; x < MB; x++)
#pragma unroll
                for (int y = 0; y < NB; y++) {
                    const v4f_t p = block_product<FA, FB>(b[u][y], a[u][x]);
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[x][y][e] = fmaf(p[e], sa[u][x] * sb[u][y][ROWS_B ? e : 0], acc[x][y][e]);
                }
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int x = 0; x < MB; x++)
#pragma unroll
            for (int y = 0; y < NB; y++) *reinterpret_cast<v4f_t *>(red[wave - 1][x * NB + y][lane]) = acc[x][y];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) {
            if (wave != 0) continue;
            v4f_t v = acc[x][y];
#pragma unroll
            for (int w = 0; w < NW - 1; w++) {
                const v4f_t o = *reinterpret_cast<const v4f_t *>(red[w][x * NB + y][lane]);
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] += o[e];
            }
            const int64_t r = m0 + 16 * x + i, c = n0 + 16 * y + 4 * q;
            if (r < g.M && c < g.N) store4<CDT>(g.C, r * g.ldc + c, g.N - c, v);
        }
}

}  // namespace mx
