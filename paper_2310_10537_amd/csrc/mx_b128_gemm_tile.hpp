// Larger products with a scale per 128 (the formula and the operand order: mx_b128_gemm.hpp).
//
// Eight waves, two on each SIMD, in KS groups of WM x WN that share the range of K; a wave owns 16 MB x 16 NB entries, a group 16 MB WM x
// 16 NB WN.  Three forms are used: 256 x 256 and 256 x 128 (one group of 4 x 2 waves, 64 x 128 or 64 x 64 entries each) and 128 x 128 (two groups
// of 2 x 2 waves, 64 x 64 entries each, half of K each: as many waves a tile where there are few tiles).
// The scaling of the partial sums is vector work, 4 instructions of 4 clocks beside each matrix instruction of 32, and a wave issues an
// instruction about every 5 clocks, so one wave on a SIMD cannot issue all that a matrix instruction wants beside it (four waves of 96 x 128 entries, operands in
// accumulation registers: 383 us for 8192 x 11008 x 4096, 351 for 2048 x 8192 x 16384 with a scale a column; eight waves: 324-341 and 262-278).  With two, one
// wave's vector work runs under the other's matrix instructions: alone on a SIMD, two waves take 33 clocks for a matrix instruction with four multiply-adds,
// 46 with eight (a matrix instruction keeps the vector pipe from others for about 14 clocks), so with a scale a column of B the vector work is the bound.
// What is left is power: the clock is at 1.8 to 1.9 GHz, and on operands of zeros the two products take 275 and 225 us.  Lines fetched into the L2 two steps ahead
// take 10 % off the time on zeros and add 3 % to it on Gaussian operands, so they are not.
// A step's matrix instructions run beside
//     the vector work:   the multiply-adds of the instruction tile three back (a ring of four results: by then it has left the pipe),
//     LDS reads:         a fragment's successor, as soon as the last instruction that reads it is on its way: a wave keeps MB fragments of
//                        A and four of B,
//     direct loads:      the stage after next, global to LDS.
// The one barrier of a step stands where all fragments of the stage in hand have been asked for (so that its buffer may be filled again); the
// first of the next stage follows behind it.
#pragma once

#include <type_traits>

#include "mx_b128_gemm.hpp"

namespace mx {

// block_product as a statement that stays where it is written.  The compiler does not know what is inside: whoever reads the result keeps 12
// instructions between (8 passes and 4), see the kernel's ring.
template <int FA, int FB>
__device__ __forceinline__ void block_product_at(v4f_t &p, const v8i_t &b, const v8i_t &a)
{
    constexpr int HA = hw_fmt(FA), HB = hw_fmt(FB);
    asm volatile("v_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0 cbsz:%3 blgp:%4" : "=&v"(p) : "v"(b), "v"(a), "n"(HB), "n"(HA) : "memory");
}

// ... with a direct load of 1 KB behind it, from base + o (a lane's bytes) to LDS byte dst + AT.  A write to M0 wants an instruction before its reader:
// the product stands there (2 % faster over eleven large products than with one of its own).
template <int FA, int FB, int AT>
__device__ __forceinline__ void block_product_and_load_at(v4f_t &p, const v8i_t &b, const v8i_t &a, uint32_t o, const uint8_t *base, uint32_t dst)
{
    constexpr int HA = hw_fmt(FA), HB = hw_fmt(FB);
    asm volatile("s_add_u32 m0, %7, %8\n\tv_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0 cbsz:%3 blgp:%4\n\tglobal_load_lds_dwordx4 %5, %6"
                 : "=&v"(p) : "v"(b), "v"(a), "n"(HB), "n"(HA), "v"(o), "s"(base), "s"(dst), "n"(AT) : "m0", "scc", "memory");
}

// a pointer that every lane of a wave has the same value of, in scalar registers
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p)
{
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return reinterpret_cast<const uint8_t *>((uint64_t)hi << 32 | lo);
}

// f(0), f(1), ..., f(N - 1) with the numbers as types
template <int N, typename F, int K = 0>
__device__ __forceinline__ void each(F f)
{
    if constexpr (K < N) {
        f(std::integral_constant<int, K>());
        each<N, F, K + 1>(f);
    }
}

constexpr int TILE_MIN_BLOCKS = 4;                    // blocks along K that a group needs: scales travel four at a time

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int WM, int WN, int KS>
__global__ __launch_bounds__(512, 2) void gemm128_tile_kernel(Gemm128 g, Bands order)
{
    static_assert(WM * WN * KS == 8 && (KS == 1 || (KS == 2 && MB % 2 == 0)) && MB >= 3, "eight waves");
    constexpr int NW = WM * WN, BM = 16 * MB * WM, BN = 16 * NB * WN, NT = MB * NB;   // of a group
    constexpr int RING = 4;                           // fragments of B in registers
    constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    constexpr int SCALE_ROWS = BM + (ROWS_B ? BN : BN / 128);
    static_assert(128 % (16 * NB) == 0 && BN % 128 == 0, "a wave's columns lie in one block");
    __shared__ __attribute__((aligned(16))) uint8_t lds_all[KS * 2 * STAGE];
    __shared__ __attribute__((aligned(16))) float scl_all[KS * 2 * 4 * SCALE_ROWS];
    const int lane = threadIdx.x & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = wave_all / NW, wave = wave_all - group * NW, tid = threadIdx.x - group * (64 * NW);
    const int wm = wave / WN, wn = wave - wm * WN;
    const int i = lane & 15, q = lane >> 4;
    uint8_t *const lds = lds_all + group * 2 * STAGE;
    float *const scl = scl_all + group * 2 * 4 * SCALE_ROWS;
    int tm, tn;
    if (!band_tile(order, (int)blockIdx.x, tm, tn)) return;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int T_all = (int)(g.K / 128), T = T_all / KS;   // blocks, and this group's: KS divides them, TILE_MIN_BLOCKS at least
    const int t_first = group * T;
    const int rows_a = (int)(g.M - m0 < BM ? g.M - m0 : BM), rows_b = (int)(g.N - n0 < BN ? g.N - n0 : BN);

    // ---- staging: load j of wave w fills rows 8 NW j + 8 w .. + 7 of the tile, lane l slot l % 8 of row l / 8.  Offsets are 32 bits from the
    // tile's first row (K below 2^24); rows beyond the matrix read its last one.
    constexpr int NJA = BM / 8 / NW, NJB = BN / 8 / NW, NJ = NJA + NJB;
    static_assert(NJA * NW * 1024 == A_BYTES, "B's stage lies behind A's");
    typedef __attribute__((address_space(3))) void lds_ptr_t;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t *)lds) + wave * 1024;
    const int s_r = wave * 8 + (lane >> 3);
    const uint32_t K32 = (uint32_t)g.K, chunk = (uint32_t)((lane & 7) ^ ((s_r >> 1) & 7)) << 4;
    const uint32_t ofs = (uint32_t)s_r * K32 + chunk;
    const uint32_t lastA = (uint32_t)(rows_a - 1) * K32 + chunk, lastB = (uint32_t)(rows_b - 1) * K32 + chunk;
    const uint8_t *const gA = uniform(g.Ae + m0 * g.K + (int64_t)t_first * 128), *const gB = uniform(g.Be + n0 * g.K + (int64_t)t_first * 128);
    auto source = [&](auto number) __attribute__((always_inline)) {               // offset of direct load k of a stage: A's, then B's (to LDS byte 1024 k NW)
        constexpr int k = decltype(number)::value, j = k < NJA ? k : k - NJA;
        const uint32_t o = ofs + (uint32_t)(8 * NW * j) * K32, last = k < NJA ? lastA : lastB;
        return o < last ? o : last;
    };
    auto load_one = [&](auto number, const uint8_t *atA, const uint8_t *atB, uint32_t dst) __attribute__((always_inline)) {
        constexpr int k = decltype(number)::value;
        const uint32_t o = source(number);
        const uint8_t *const base = k < NJA ? atA : atB;
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(o), "s"(base), "s"(dst), "n"(k * NW * 1024) : "m0", "scc", "memory");
    };
    // ---- scales, four blocks at a time: those of blocks first(G) .. + 3, G = 0, 1, ...; the last group of a row is its last four
    auto first = [&](int G) { return 4 * G + 4 <= T ? 4 * G : T - 4; };
    auto scale_row = [&](int t) { return scl + (((t >> 2) & 1) * 4 + t - first(t >> 2)) * SCALE_ROWS; };          // block t's, in [2][4]
    // thread r: row r of A, beyond them the blocks of B's columns; or (ROWS_B) row r - BM of B, in two goes where the threads are fewer than the rows
    constexpr int NS = (SCALE_ROWS + 64 * NW - 1) / (64 * NW);
    const float *pS[NS];
#pragma unroll
    for (int j = 0; j < NS; j++) {
        const int r = j * 64 * NW + tid, rb = r - BM;
        if (rb < 0) {
            pS[j] = g.As + ((m0 + (r < rows_a ? r : rows_a - 1)) >> g.a_shift) * T_all + t_first;
        } else if (ROWS_B) {
            pS[j] = g.Bs + (n0 + (rb < rows_b ? rb : rows_b - 1)) * T_all + t_first;
        } else {
            const int64_t blk = (n0 >> 7) + (rb < BN / 128 ? rb : 0), last = (g.N - 1) >> 7;
            pS[j] = g.Bs + (blk < last ? blk : last) * T_all + t_first;
        }
    }
    float sv[NS][4];
    auto fetch_scales = [&](int G) __attribute__((always_inline)) {
        const int f = first(G);
#pragma unroll
        for (int j = 0; j < NS; j++)
            if (j * 64 * NW + tid < SCALE_ROWS) __builtin_memcpy(sv[j], __builtin_assume_aligned(pS[j] + f, 4), 16);
    };
    auto park_scales = [&](int G) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NS; j++)
            if (j * 64 * NW + tid < SCALE_ROWS) {
#pragma unroll
                for (int e = 0; e < 4; e++) scl[((G & 1) * 4 + e) * SCALE_ROWS + j * 64 * NW + tid] = sv[j][e];
            }
    };

    const int ra0 = (wm * 16 * MB + i) * 128 + ((q ^ ((i >> 1) & 7)) << 4);
    const int rb0 = A_BYTES + (wn * 16 * NB + i) * 128 + ((q ^ ((i >> 1) & 7)) << 4);
    auto frag = [&](int buf, int at, int x) __attribute__((always_inline)) {
        const uint4 lo = *reinterpret_cast<const uint4 *>(lds + buf + at + x * 2048);
        const uint4 hi = *reinterpret_cast<const uint4 *>(lds + buf + (at ^ 64) + x * 2048);
        return v8i_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
    };

    v4f_t acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; x++)
#pragma unroll
        for (int y = 0; y < NB; y++) acc[x][y] = v4f_t{0.f, 0.f, 0.f, 0.f};
    v8i_t a[MB], b[RING];
    float s[MB], sn[MB];
    v4f_t p[4], bs[2];
    const int sa0 = wm * 16 * MB + i, sb0 = BM + wn * 16 * NB + 4 * q, sb_tile = BM + ((wn * 16 * NB) >> 7);

    // One instruction tile: its 128 products, and the multiply-adds of the one three back (with scales f).  An empty statement in front keeps
    // those behind the instructions issued so far: from a result's instruction to its first reader there are two others and three times four multiply-adds.
    auto scale_tile = [&](auto tile, const float (&f)[MB]) __attribute__((always_inline)) {
        constexpr int k = decltype(tile)::value, x = k % MB, y = k / MB;
#pragma unroll
        for (int e = 0; e < 4; e++) acc[x][y][e] = fmaf(p[k & 3][e], ROWS_B ? f[x] * bs[y & 1][e] : f[x], acc[x][y][e]);
        asm volatile("" : "+v"(acc[x][y]));           // (here, not where the sum is wanted: the ring's place is wanted before)
    };
    auto tile = [&](auto number, const float *sc, const float (&f)[MB], auto also, auto beside, auto product) __attribute__((always_inline)) {
        constexpr int k = decltype(number)::value, x = k % MB, y = k / MB, back = (k + NT - 3) % NT;
        if constexpr (decltype(also)::value) asm volatile("" : "+v"(p[back & 3]));
        product(number, p[k & 3], b[y % RING], a[x]);
        beside(number);
        if constexpr (decltype(also)::value) scale_tile(std::integral_constant<int, back>(), f);
        if constexpr (ROWS_B && x == 2) bs[(y + 1) & 1] = *reinterpret_cast<const v4f_t *>(sc + 16 * ((y + 1) % NB));
        __builtin_amdgcn_sched_barrier(0);
    };
    auto alone = [](auto, v4f_t &to, const v8i_t &fb, const v8i_t &fa) __attribute__((always_inline)) { block_product_at<FA, FB>(to, fb, fa); };
    constexpr std::true_type with;
    constexpr std::false_type without;
    static_assert(NT % 4 == 0, "the ring's places repeat from step to step");

    // ---- stages 0 and 1, scales of group 0; the registers of step 0
    fetch_scales(0);
    each<NJ>([&](auto k) { load_one(k, gA, gB, lds0); });
    each<NJ>([&](auto k) { load_one(k, gA + 128, gB + 128, lds0 + STAGE); });
    park_scales(0);
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NJ) : "memory");
    __syncthreads();
#pragma unroll
    for (int x = 0; x < MB; x++) a[x] = frag(0, ra0, x);
#pragma unroll
    for (int y = 0; y < RING; y++) b[y] = frag(0, rb0, y);
#pragma unroll
    for (int x = 0; x < MB; x++) s[x] = scale_row(0)[sa0 + 16 * x] * (ROWS_B ? 1.0f : scale_row(0)[sb_tile]);
    if constexpr (ROWS_B) bs[0] = *reinterpret_cast<const v4f_t *>(scale_row(0) + sb0);

    // A trip of the loop runs from the barrier of step t to that of step t + 1: the tiles from FRONT on of step t, then the first FRONT of the
    // next.  By then all fragments of the step in hand have been asked for; the first of the next follows.
    constexpr int FRONT = RING == NB ? 2 * MB : 5 * MB - 1;
    static_assert(NT - FRONT >= NJ && NT - FRONT >= 6, "a direct load beside each of the instructions behind it");
    // in front of the barrier: (RING < NB) a column's fragment makes room for the one RING columns on
    auto front = [&](int cur) {
        return [&, cur](auto number) __attribute__((always_inline)) {
            constexpr int k = decltype(number)::value, x = k % MB, y = k / MB;
            if constexpr (RING < NB && x == MB - 1) b[y % RING] = frag(cur, rb0, y + RING);
        };
    };
    each<3>([&](auto k) { tile(k, scale_row(0) + sb0, s, without, front(0), alone); });
    asm volatile("s_nop 15" : "+v"(p[0]));            // (nothing stands between these three and the first multiply-adds)
    each<FRONT - 3>([&](auto d) { tile(std::integral_constant<int, 3 + decltype(d)::value>(), scale_row(0) + sb0, s, with, front(0), alone); });
    for (int t = 0; t + 1 < T; t++) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if ((t & 3) == 2 && t + 2 < T) park_scales((t >> 2) + 1);
        __syncthreads();
        if ((t & 3) == 1 && t + 3 < T) fetch_scales((t >> 2) + 1);
        const int nxt = ((t + 1) & 1) * STAGE;        // the buffer of step t + 1
        const uint32_t dst = lds0 + (t & 1) * STAGE;  // where the stage after it goes (behind the last: that one again)
        const int64_t at = (int64_t)(t + 2 < T ? t + 2 : T - 1) * 128;
        const uint8_t *const atA = gA + at, *const atB = gB + at;
        const float *const sc = scale_row(t) + sb0, *const sc1 = scale_row(t + 1);
        float sb1 = 1.0f;
        auto fill = [&](auto number) __attribute__((always_inline)) {
            constexpr int k = decltype(number)::value, x = k % MB, y = k / MB, d = k - FRONT;
            if constexpr (RING == NB && (d == 2 || d == 5)) b[d / 3] = frag(nxt, rb0, d / 3);     // the first two columns' fragments fell free before
            if constexpr (x == MB - 1) b[y % RING] = frag(nxt, rb0, y % RING);
            if constexpr (y == NB - 1) a[x] = frag(nxt, ra0, x);
            if constexpr (y == NB - 1) sn[x] = sc1[sa0 + 16 * x];
            if constexpr (!ROWS_B && k == NT - MB) sb1 = sc1[sb_tile];
        };
        auto and_load = [&](auto number, v4f_t &to, const v8i_t &fb, const v8i_t &fa) __attribute__((always_inline)) {
            constexpr int d = decltype(number)::value - FRONT;
            if constexpr (d < NJ) block_product_and_load_at<FA, FB, d * NW * 1024>(to, fb, fa, source(std::integral_constant<int, d>()), d < NJA ? atA : atB, dst);
            else alone(number, to, fb, fa);
        };
        each<NT - FRONT>([&](auto d) {
            constexpr int k = FRONT + decltype(d)::value;
            const std::integral_constant<int, k> number;
            const float *const of = ROWS_B && k / MB == NB - 1 ? sc1 + sb0 : sc;  // (the scales fetched ahead in the last column are the next step's)
            tile(number, of, s, with, fill, and_load);
        });
        each<FRONT>([&](auto k) {
            if constexpr (!ROWS_B && k() < MB) {
                constexpr int x = decltype(k)::value;
                tile(k, sc1 + sb0, x < 3 ? s : sn, with, [&](auto n) { sn[x] *= sb1; front(nxt)(n); }, alone);
            } else {
                if constexpr (k() < 3) tile(k, sc1 + sb0, s, with, front(nxt), alone);
                else tile(k, sc1 + sb0, sn, with, front(nxt), alone);
            }
        });
#pragma unroll
        for (int x = 0; x < MB; x++) s[x] = sn[x];
    }
    each<NT - FRONT>([&](auto d) { tile(std::integral_constant<int, FRONT + decltype(d)::value>(), scale_row(T - 1) + sb0, s, with, [](auto) {}, alone); });
    each<3>([&](auto k) {
        asm volatile("s_nop 3" : "+v"(p[(NT - 3 + k()) & 3]));
        scale_tile(std::integral_constant<int, NT - 3 + k()>(), s);
    });
    // the last direct loads must have landed before this LDS is used again, here or by another work-group
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (KS == 2) {
        // each group finishes half of a wave's rows: the others' sums go to the other group by way of LDS; first group + second group
        float *const mine = reinterpret_cast<float *>(lds_all) + (group * NW + wave) * (NT / 2) * 256, *const other = reinterpret_cast<float *>(lds_all) + ((1 - group) * NW + wave) * (NT / 2) * 256;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < MB / 2; x++)
#pragma unroll
            for (int y = 0; y < NB; y++) *reinterpret_cast<v4f_t *>(mine + ((x * NB + y) * 64 + lane) * 4) = group ? acc[x][y] : acc[x + MB / 2][y];
        __syncthreads();
#pragma unroll
        for (int x = 0; x < MB / 2; x++)
#pragma unroll
            for (int y = 0; y < NB; y++) {
                const v4f_t o = *reinterpret_cast<const v4f_t *>(other + ((x * NB + y) * 64 + lane) * 4), v = group ? acc[x + MB / 2][y] : acc[x][y];
#pragma unroll
                for (int e = 0; e < 4; e++) acc[x][y][e] = group ? o[e] + v[e] : v[e] + o[e];
            }
        store_rows<CDT, MB / 2, NB>(g, acc, m0 + wm * 16 * MB + group * 8 * MB, n0 + wn * 16 * NB, i, q);
    } else {
        store_rows<CDT, MB, NB>(g, acc, m0 + wm * 16 * MB, n0 + wn * 16 * NB, i, q);
    }
}

template <int FA, int FB, int CDT, bool ROWS_B, int MB, int NB, int WM, int WN, int KS>
static hipError_t launch_tile(const Gemm128 &g, hipStream_t st)
{
    constexpr int BM = 16 * MB * WM, BN = 16 * NB * WN;
    const int64_t tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
    if (tm > ((int64_t)1 << 22) / tn) return hipErrorNotSupported;     // (the runtime counts a grid's threads in 32 bits)
    // a work-group of 256 x 256 has a compute unit to itself, so 32 of them run on an XCD: 5 rows by 6 to 7 columns fetch least (8192 x 11008 x 4096: 2.21
    // PFLOP/s in bands of 5, 2.20 of 6, 2.14 of 4; 16384 x 8192 x 2048: 2.13, 2.09, 2.00)
    const Bands order = bands(tm, tn, BM == 256 && BN == 256 ? 5 : 6);
    hipLaunchKernelGGL((gemm128_tile_kernel<FA, FB, CDT, ROWS_B, MB, NB, WM, WN, KS>), dim3(8 * order.per_xcd), dim3(512), 0, st, g, order);
    return hipGetLastError();
}

}  // namespace mx
