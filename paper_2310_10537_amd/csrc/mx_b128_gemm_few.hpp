// The product of mx_b128_gemm.hpp for few rows of A, where reading B is all that costs: each byte of B is wanted once, so it goes
// straight to registers; and for products of so few entries that one round of small work-groups covers them, where the way along K is all that costs.
// A work-group has 16 MB rows and 16 NB columns; its eight waves take an eighth of the blocks along K each, with AHEAD blocks on
// their way, and their partial sums are added in a fixed order through LDS.  A load takes 64 consecutive bytes of 16 rows; rows of A that do
// not exist are not loaded (one row: half of the load path's work).  1 x 11008 x 4096: 11.4 us, 3.9 TB/s of weights; 1 x 28672 x 8192: 48.6 us, 4.8 TB/s.
#pragma once

#include "mx_b128_gemm.hpp"

namespace mx {

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int AHEAD>
__global__ __launch_bounds__(512) void gemm128_few_kernel(Gemm128 g)
{
    constexpr int NW = 8;
    __shared__ __attribute__((aligned(16))) float red[NW][MB * NB][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * NB), m0 = (int64_t)blockIdx.y * (16 * MB);
    const int T = (int)(g.K / 128);
    // blocks of this wave: an eighth each, the first T % 8 waves one more
    const int base = T / NW, extra = T % NW;
    const int t0 = wave * base + (wave < extra ? wave : extra), t1 = t0 + base + (wave < extra ? 1 : 0);

    const uint8_t *pA[MB], *pB[NB];
    const float *sA[MB], *sB[NB];
    bool on[MB];                                      // rows beyond M are not read: zeros
#pragma unroll
    for (int x = 0; x < MB; x++) {
        const int64_t row = m0 + 16 * x + i;
        on[x] = row < g.M;
        pA[x] = g.Ae + (on[x] ? row : 0) * g.K + 16 * q;
        sA[x] = g.As + ((on[x] ? row : 0) >> g.a_shift) * T;
    }
#pragma unroll
    for (int y = 0; y < NB; y++) {                    // columns beyond N: the last one, not stored
        const int64_t col = n0 + 16 * y + i < g.N ? n0 + 16 * y + i : g.N - 1;
        pB[y] = g.Be + col * g.K + 16 * q;
        sB[y] = g.Bs + (ROWS_B ? 0 : ((n0 + 16 * y < g.N ? n0 + 16 * y : g.N - 1) >> 7) * T);
    }
    v4f_t acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) acc[x][y] = v4f_t{0.f, 0.f, 0.f, 0.f};

    struct Block { uint4 a[MB][2], b[NB][2]; float sa[MB], sb[NB][ROWS_B ? 4 : 1]; };
    auto request = [&](Block &o, int t) __attribute__((always_inline)) {
        const int64_t at = (int64_t)t * 128;
#pragma unroll
        for (int y = 0; y < NB; y++) { o.b[y][0] = ld16_nt(pB[y] + at); o.b[y][1] = ld16_nt(pB[y] + at + 64); }
#pragma unroll
        for (int x = 0; x < MB; x++) {
            o.a[x][0] = o.a[x][1] = make_uint4(0, 0, 0, 0);
            o.sa[x] = 0.0f;
            if (on[x]) { o.a[x][0] = ld16(pA[x] + at); o.a[x][1] = ld16(pA[x] + at + 64); o.sa[x] = sA[x][t]; }
        }
#pragma unroll
        for (int y = 0; y < NB; y++) {
            if constexpr (ROWS_B) {                   // a scale for each of the lane's four columns
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int64_t c = n0 + 16 * y + 4 * q + e;
                    o.sb[y][e] = g.Bs[(c < g.N ? c : g.N - 1) * T + t];
                }
            } else {
                o.sb[y][0] = sB[y][t];
            }
        }
    };
    auto add = [&](const Block &o) __attribute__((always_inline)) {
        auto frag = [](const uint4 (&v)[2]) { return v8i_t{(int)v[0].x, (int)v[0].y, (int)v[0].z, (int)v[0].w, (int)v[1].x, (int)v[1].y, (int)v[1].z, (int)v[1].w}; };
#pragma unroll
        for (int x = 0; x < MB; x++)
#pragma unroll
            for (int y = 0; y < NB; y++) {
                const v4f_t p = block_product<FA, FB>(frag(o.b[y]), frag(o.a[x]));
#pragma unroll
                for (int e = 0; e < 4; e++) acc[x][y][e] = fmaf(p[e], o.sa[x] * o.sb[y][ROWS_B ? e : 0], acc[x][y][e]);
            }
    };
    if (t0 < t1) {
        // a ring of AHEAD blocks on their way
        Block ring[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
            if (t0 + u < t1) request(ring[u], t0 + u);
        for (int t = t0; t < t1; t += AHEAD) {
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                if (t + u < t1) add(ring[u]);
                if (t + u + AHEAD < t1) request(ring[u], t + u + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) *reinterpret_cast<v4f_t *>(red[wave][x * NB + y][lane]) = acc[x][y];
    __syncthreads();
    // each wave adds up and stores its share of the tiles
    for (int k = wave; k < MB * NB; k += NW) {
        v4f_t v = *reinterpret_cast<const v4f_t *>(red[0][k][lane]);
#pragma unroll
        for (int w = 1; w < NW; w++) {
            const v4f_t o = *reinterpret_cast<const v4f_t *>(red[w][k][lane]);
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] += o[e];
        }
        const int x = k / NB, y = k - x * NB;
        const int64_t r = m0 + 16 * x + i, c = n0 + 16 * y + 4 * q;
        if (r < g.M && c < g.N) store4<CDT>(g.C, r * g.ldc + c, g.N - c, v);
    }
}

}  // namespace mx
