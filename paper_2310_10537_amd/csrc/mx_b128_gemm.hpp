// C = A . B^T for 8-bit operands with a Float32 scale for each block of 128 along K:
//     C[m][n] = sum over blocks b of (sum_{j in b} a[m][j] b[n][j]) * (sA[m][b] * sB[n][b]),
// A's scales one a row and block, or one for 128 rows and a block (ROWS_A is a run-time shift); B's the same.
//
// The 16 x 16 x 128 matrix instruction adds exactly the products of one block, from zero, so a scale meets its partial sum in one Float32
// multiply-add per entry and block.  That vector work decides the layout: accumulators have to be in the vector
// registers (the instructions that scale them cannot reach the accumulation registers), 256 of them a lane at most, so
// a 256 x 256 tile takes eight waves of 64 x 128 entries (128 accumulators a lane), two on each SIMD (mx_b128_gemm_tile.hpp).
// The B fragment goes first: a lane (i, q) then holds row i of A and four consecutive columns 4q .. 4q + 3, so the scale of A is one
// number a lane and 16-row block, and where B has a scale for 128 columns that one is the same for the whole wave (its columns lie in one
// block of 128): one product a lane, block and 16 rows, all else is multiply-adds.  With a scale a column of B four products and four multiply-adds.
#pragma once

#include "mx_b128.hpp"
#include "mx_gemm_frag.hpp"
#include "mx_launch.hpp"

namespace mx {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float v4f_t __attribute__((ext_vector_type(4)));

struct Gemm128 {
    int64_t M, N, K;
    const uint8_t *Ae, *Be;
    const float *As, *Bs;
    int a_shift, b_shift;         // 0: a scale a row, 7: one for 128 rows
    void *C;
    int64_t ldc;
};

// Order of the tiles of C, for a grid of any size.  Work-groups are dealt round-robin to the 8 XCDs, each with its own L2, and the 32 or 64 that an XCD
// works on at a time walk K in step: what they fetch per step is a slab of A for each of their tile rows and one of B for each tile
// column.  So the tiles are numbered in bands of h rows, column by column, and each XCD takes an eighth of the numbers: its running tiles
// form a patch of h rows.
struct Bands { int tiles_m, tiles_n, h, per_xcd; };
inline Bands bands(int64_t tiles_m, int64_t tiles_n, int h)
{
    return Bands{(int)tiles_m, (int)tiles_n, (int)(tiles_m < h ? tiles_m : h), (int)((tiles_m * tiles_n + 7) / 8)};
}
// tile of work-group b; false when it has none
__device__ __forceinline__ bool band_tile(const Bands &r, int b, int &tm, int &tn)
{
    const int at = (b & 7) * r.per_xcd + (b >> 3), area = r.h * r.tiles_n;
    if (at >= r.tiles_m * r.tiles_n) return false;
    const int band = at / area, in = at - band * area, left = r.tiles_m - band * r.h, h = left < r.h ? left : r.h;
    tn = in / h;
    tm = band * r.h + in - tn * h;
    return true;
}

// 128 products of each of 16 x 16 entries, from zero (unit scales: plain products)
template <int FA, int FB>
__device__ __forceinline__ v4f_t block_product(const v8i_t &b, const v8i_t &a)
{
    constexpr int HA = hw_fmt(FA), HB = hw_fmt(FB);   // must reach the builtin as literal constants
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, v4f_t{0.f, 0.f, 0.f, 0.f}, HB, HA, 0, 0, 0, 0);
}

// N consecutive values of a row of C to it, as far as they lie inside (left: columns that do).  Rows start anywhere: the vector stores assume the
// alignment of an element only.
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store4_f32(float *o, int64_t left, const v4f_t &v)
{
    if (left >= 4) {
        *reinterpret_cast<f32x4_at4 *>(o) = f32x4_at4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < left) o[i] = v[i];
    }
}
template <int ND>
__device__ __forceinline__ void store_bf16(uint16_t *o, int64_t left, const uint32_t (&d)[ND])
{
    if (left >= 2 * ND) {
        if constexpr (ND == 4) *reinterpret_cast<u32x4_at2 *>(o) = u32x4_at2{d[0], d[1], d[2], d[3]};
        else *reinterpret_cast<u32x2_at2 *>(o) = u32x2_at2{d[0], d[1]};
    } else {
#pragma unroll
        for (int i = 0; i < 2 * ND - 1; i++)
            if (i < left) o[i] = (uint16_t)(d[i >> 1] >> (16 * (i & 1)));
    }
}
// one instruction tile's four columns of a lane's row
template <int CDT>
__device__ __forceinline__ void store4(void *__restrict__ C, int64_t at, int64_t left, const v4f_t &v)
{
    if constexpr (CDT == DT_F32) {
        store4_f32(static_cast<float *>(C) + at, left, v);
    } else {
        const uint32_t d[2] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        store_bf16<2>(static_cast<uint16_t *>(C) + at, left, d);
    }
}
// A wave's MX x NY instruction tiles, rows from row0 and columns from col0 on.  bf16: the lanes q and q ^ 1 of a row hold neighbouring column
// groups; they trade between two tiles (the row swap of the lane permutes does exactly that), so that each stores eight columns: 64
// contiguous bytes a row and instruction.
template <int CDT, int MX, int NY, int MROWS>
__device__ __forceinline__ void store_rows(const Gemm128 &g, const v4f_t (&acc)[MROWS][NY], int64_t row0, int64_t col0, int i, int q)
{
#pragma unroll
    for (int x = 0; x < MX; x++) {
        const int64_t r = row0 + 16 * x + i;
        if constexpr (CDT == DT_F32) {
#pragma unroll
            for (int y = 0; y < NY; y++) {
                const int64_t c = col0 + 16 * y + 4 * q;
                if (r < g.M && c < g.N) store4<CDT>(g.C, r * g.ldc + c, g.N - c, acc[x][y]);
            }
        } else {
#pragma unroll
            for (int y = 0; y < NY; y += 2) {
                const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(acc[x][y][0], acc[x][y][1]), pack_bf16(acc[x][y + 1][0], acc[x][y + 1][1]), false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(acc[x][y][2], acc[x][y][3]), pack_bf16(acc[x][y + 1][2], acc[x][y + 1][3]), false, false);
                const uint32_t d[4] = {lo[0], hi[0], lo[1], hi[1]};
                const int64_t c = col0 + 16 * y + 16 * (q & 1) + 4 * (q & 2);
                if (r < g.M && c < g.N) store_bf16<4>(static_cast<uint16_t *>(g.C) + r * g.ldc + c, g.N - c, d);
            }
        }
    }
}
// Work-group tile BM x BN: WM x WN waves of 16 MB x 16 NB entries.  K in steps of one block through two LDS buffers, laid out as in the MX
// kernels (128 bytes a row, chunk c of row r in slot c ^ ((r >> 1) & 7): direct loads fill any permutation of 16-byte slots, and the
// operand reads meet no bank twice).  Rows beyond M and columns beyond N read the last valid one and are not stored.
// Scales travel four blocks at a time, 16 bytes a row, by way of registers into [block][row] in LDS.
template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void gemm128_kernel(Gemm128 g, Bands order)
{
    constexpr int NW = WM * WN, BM = 16 * MB * WM, BN = 16 * NB * WN, NTHREADS = 64 * NW;
    constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    constexpr int SCALE_ROWS = BM + (ROWS_B ? BN : 0);
    static_assert(ROWS_B || 128 % (16 * NB) == 0, "a wave's columns lie in one block");
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * STAGE];
    __shared__ __attribute__((aligned(16))) float scl[2][4][SCALE_ROWS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN;
    const int i = lane & 15, q = lane >> 4;
    int tm, tn;
    if (!band_tile(order, (int)blockIdx.x, tm, tn)) return;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int T = (int)(g.K / 128);

    // ---- staging: load j of wave w fills rows (j NW + w) * 8 .. + 7 of the tile, lane l slot l % 8 of row l / 8
    constexpr int NJA = BM / 8 / NW, NJB = BN / 8 / NW;
    static_assert(NJA * 8 * NW == BM && NJB * 8 * NW == BN, "whole loads");
    typedef __attribute__((address_space(3))) void lds_ptr_t;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t *)lds) + wave * 1024;
    const uint8_t *pA[NJA], *pB[NJB];
#pragma unroll
    for (int j = 0; j < NJA; j++) {
        const int r = (j * NW + wave) * 8 + (lane >> 3);
        const int64_t row = m0 + r < g.M ? m0 + r : g.M - 1;
        pA[j] = g.Ae + row * g.K + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
    }
#pragma unroll
    for (int j = 0; j < NJB; j++) {
        const int r = (j * NW + wave) * 8 + (lane >> 3);
        const int64_t row = n0 + r < g.N ? n0 + r : g.N - 1;
        pB[j] = g.Be + row * g.K + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
    }
    auto stage = [&](int t, int buf) {
#pragma unroll
        for (int j = 0; j < NJA; j++) {
            const uint8_t *p = pA[j] + (int64_t)t * 128;
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds0 + buf * STAGE + j * NW * 1024) : "m0", "memory");
        }
#pragma unroll
        for (int j = 0; j < NJB; j++) {
            const uint8_t *p = pB[j] + (int64_t)t * 128;
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds0 + buf * STAGE + A_BYTES + j * NW * 1024) : "m0", "memory");
        }
    };
    // ---- scales of blocks 4G .. 4G + 3: thread r those of row r of A, then of B
    constexpr int NS = (SCALE_ROWS + NTHREADS - 1) / NTHREADS;
    const float *pS[NS];
    bool s_on[NS];
#pragma unroll
    for (int j = 0; j < NS; j++) {
        const int r = j * NTHREADS + tid;
        s_on[j] = r < SCALE_ROWS;
        const bool of_a = r < BM;
        const int64_t row = of_a ? (m0 + r < g.M ? m0 + r : g.M - 1) : (n0 + r - BM < g.N ? n0 + r - BM : g.N - 1);
        pS[j] = of_a ? g.As + (row >> g.a_shift) * T : g.Bs + row * T;
    }
    float sv[NS][4];
    auto fetch_scales = [&](int G) {
#pragma unroll
        for (int j = 0; j < NS; j++) {
            if (!s_on[j]) continue;
            const float *p = pS[j] + 4 * G;
            if (4 * G + 4 <= T) {
                __builtin_memcpy(sv[j], __builtin_assume_aligned(p, 4), 16);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) sv[j][e] = 4 * G + e < T ? p[e] : 0.0f;
            }
        }
    };
    auto park_scales = [&](int G) {
#pragma unroll
        for (int j = 0; j < NS; j++)
            if (s_on[j]) {
#pragma unroll
                for (int e = 0; e < 4; e++) scl[G & 1][e][j * NTHREADS + tid] = sv[j][e];
            }
    };
    const int64_t nb = (n0 + wn * 16 * NB) >> 7, nb_last = (g.N - 1) >> 7;
    const float *const pSB = g.Bs + (nb < nb_last ? nb : nb_last) * T;      // (!ROWS_B) this wave's scales of B

    const int ra0 = (wm * 16 * MB + i) * 128 + ((q ^ ((i >> 1) & 7)) << 4);
    const int rb0 = (wn * 16 * NB + i) * 128 + ((q ^ ((i >> 1) & 7)) << 4);
    auto frag = [&](const uint8_t *buf, int ofs, int x) {
        const uint4 lo = *reinterpret_cast<const uint4 *>(buf + ofs + x * 2048);
        const uint4 hi = *reinterpret_cast<const uint4 *>(buf + (ofs ^ 64) + x * 2048);
        return v8i_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };

    v4f_t acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) acc[x][y] = v4f_t{0.f, 0.f, 0.f, 0.f};

    if (T > 0) {
        fetch_scales(0);
        stage(0, 0);
        park_scales(0);
    }
    for (int t = 0; t < T; t++) {
        // stage t has landed, its scales are parked, and every wave has done with the other buffer
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < T) stage(t + 1, (t + 1) & 1);
        const int G = t >> 2;
        const bool next_scales = (t & 3) == 0 && 4 * (G + 1) < T;
        if (next_scales) fetch_scales(G + 1);
        const uint8_t *bufA = lds + (t & 1) * STAGE, *bufB = bufA + A_BYTES;
        const float *sc = scl[G & 1][t & 3];
        v8i_t a[MB];
        float s[MB];
#pragma unroll
        for (int x = 0; x < MB; x++) { a[x] = frag(bufA, ra0, x); s[x] = sc[wm * 16 * MB + 16 * x + i]; }
        if constexpr (!ROWS_B) {
            const float sb = pSB[t];
#pragma unroll
            for (int x = 0; x < MB; x++) s[x] *= sb;
        }
        v4f_t p[2][MB];
        {
            const v8i_t b = frag(bufB, rb0, 0);
#pragma unroll
            for (int x = 0; x < MB; x++) p[0][x] = block_product<FA, FB>(b, a[x]);
        }
#pragma unroll
        for (int y = 0; y < NB; y++) {
            if (y + 1 < NB) {
                const v8i_t b = frag(bufB, rb0, y + 1);
#pragma unroll
                for (int x = 0; x < MB; x++) p[(y + 1) & 1][x] = block_product<FA, FB>(b, a[x]);
            }
            if constexpr (ROWS_B) {
                const float4 f = *reinterpret_cast<const float4 *>(sc + BM + wn * 16 * NB + 16 * y + 4 * q);
                const v4f_t sb = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int x = 0; x < MB; x++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[x][y][e] = fmaf(p[y & 1][x][e], s[x] * sb[e], acc[x][y][e]);
            } else {
#pragma unroll
                for (int x = 0; x < MB; x++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[x][y][e] = fmaf(p[y & 1][x][e], s[x], acc[x][y][e]);
            }
        }
        if (next_scales) park_scales(G + 1);
    }

    store_rows<CDT, MB, NB>(g, acc, m0 + wm * 16 * MB, n0 + wn * 16 * NB, i, q);
}

}  // namespace mx
