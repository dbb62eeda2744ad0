// Casts to 8-bit floating point with one Float32 scale for each block of 128 elements, or each 128 x 128 tile
// (arithmetic in mx_b128.hpp).  All are bound by memory: 2 or 4 bytes read and 1 byte + 4/128 (4/16384) written
// per element.
//
// 8192 x 8192 bf16: rows 33.9 us (6.0 TB/s), tiles 33.0 (6.2), along dimension 0 38.7 and 37.0 (5.2, 5.5); 11008 x 4096 Float32 in tiles 37.5 (6.0).
//   cast128_row_kernel    1 x 128 blocks along the rows.  bf16: 16 lanes of 8 elements hold a block, Float32: 32
//       lanes of 4 (one 16-byte load each), four loads in flight; the block maximum is a chain of DPP row
//       operations.  Output positions are one run over all rows, filled up to whole blocks.
//   cast128_tile_kernel   128 x 128 tiles, codes in the source's order.  A work-group holds the tile in
//       registers: the maximum needs all of it before the first code can be written, and LDS would only add traffic.
//   cast128_col_kernel    blocks (or tiles) along dimension 0, written as the cast of the transpose.  The tile
//       passes through LDS, where each row block of 32 rows is rotated by a quarter of the banks so that the column reads
//       (16 columns x 4 row blocks per wave) meet no bank twice; four lanes then hold a column's block and write its 128 bytes.
#include "mx_b128.hpp"
#include "mx_launch.hpp"

namespace mx {

// The 16 bytes at element `at` of which n elements lie inside the row, as they lie in memory (the rest is zero).
template <int DT>
__device__ __forceinline__ uint4 load16(const void *__restrict__ src, int64_t at, int n)
{
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, ES = DT == DT_BF16 ? 2 : 4;
    const uint8_t *g = static_cast<const uint8_t *>(src) + at * ES;
    if (n == EPL) return ld16_nt(g);
    uint32_t h[EPL];
#pragma unroll
    for (int i = 0; i < EPL; i++) h[i] = i >= n ? 0u : DT == DT_BF16 ? (uint32_t)reinterpret_cast<const uint16_t *>(g)[i] : reinterpret_cast<const uint32_t *>(g)[i];
    if constexpr (DT == DT_BF16) return make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
    else return make_uint4(h[0], h[1], h[2], h[3]);
}
// ... as Float32 bit patterns
template <int DT>
__device__ __forceinline__ void widen(const uint4 &t, uint32_t (&v)[DT == DT_BF16 ? 8 : 4])
{
    const uint32_t d[4] = {t.x, t.y, t.z, t.w};
    if constexpr (DT == DT_BF16) {
        widen_bf16<4>(d, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = d[i];
    }
}
// The largest magnitude in 16-byte pieces, as a Float32 bit pattern; bf16 stays packed (half of a 32-bit maximum's work)
template <int DT, int N>
__device__ __forceinline__ uint32_t pieces_max(const uint4 (&t)[N])
{
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < N; p++) {
        const uint32_t d[4] = {t[p].x, t[p].y, t[p].z, t[p].w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (DT == DT_BF16) {
                m = pk_absmax(m, d[i]);
            } else {
                const uint32_t k = d[i] & 0x7FFFFFFFu;
                m = m > k ? m : k;
            }
        }
    }
    return DT == DT_BF16 ? pk_hmax(m) << 16 : m;
}

constexpr int ROW128_CHUNKS = 4;

// units of EPL elements, the rows filled up to whole blocks; units_per_row is a multiple of a block's 128 / EPL lanes, so a block never
// straddles the end of what the launch covers and every lane of it takes part in its maximum
struct Rows128 {
    FastDiv units_per_row;
    int64_t cols, ld;
    uint32_t n_units;
};

template <int FMT, int DT>
__global__ __launch_bounds__(256) void cast128_row_kernel(const void *__restrict__ src, Rows128 geom, uint8_t *__restrict__ elems, float *__restrict__ scales)
{
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, LPB = BLOCK128 / EPL;
    fp8_saturate_mode();
    const uint32_t u0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * ROW128_CHUNKS) + (threadIdx.x & 63);
    uint4 d[ROW128_CHUNKS];
#pragma unroll
    for (int c = 0; c < ROW128_CHUNKS; c++) {
        const uint32_t u = u0 + c * 64;
        int64_t at = 0;
        int n = 0;
        if (u < geom.n_units) {
            const uint32_t r = geom.units_per_row(u);
            const int64_t col = (int64_t)(u - r * geom.units_per_row.d) * EPL, left = geom.cols - col;
            n = left >= EPL ? EPL : left > 0 ? (int)left : 0;
            at = (int64_t)r * geom.ld + col;
        }
        d[c] = load16<DT>(src, at, n);
    }
#pragma unroll
    for (int c = 0; c < ROW128_CHUNKS; c++) {
        const uint32_t u = u0 + c * 64;
        auto group = [](uint32_t m) { return LPB == 16 ? row16_max(m) : row32_max(m); };
        uint32_t v[EPL], out[EPL / 4];
        widen<DT>(d[c], v);
        const uint4 one[1] = {d[c]};
        uint32_t amax = group(pieces_max<DT, 1>(one));
        float f;
        if (amax < 0x7F800000u) {
            f = b128_factor<FMT>(amax);
            b128_convert<FMT, EPL>(v, f, out);
        } else {                                      // (every lane of the block)
            f = b128_factor<FMT>(group(finite_max(v)));
            b128_convert_any<FMT, EPL>(v, f, out);
        }
        if (u < geom.n_units) {
            uint8_t *o = elems + (int64_t)u * EPL;
            if constexpr (EPL == 8) *reinterpret_cast<uint2 *>(o) = make_uint2(out[0], out[1]);
            else *reinterpret_cast<uint32_t *>(o) = out[0];
            if ((threadIdx.x & (LPB - 1)) == 0) scales[u / LPB] = 1.0f / f;
        }
    }
}

// The maximum of a work-group of 256, in every thread.  `slot`: four dwords of LDS that nobody else uses.
__device__ __forceinline__ uint32_t group256_max(uint32_t m, uint32_t *slot)
{
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = m;
    __syncthreads();
    const uint32_t a = slot[0] > slot[1] ? slot[0] : slot[1], b = slot[2] > slot[3] ? slot[2] : slot[3];
    return a > b ? a : b;
}

template <int FMT, int DT>
__global__ __launch_bounds__(256) void cast128_tile_kernel(const void *__restrict__ src, int64_t rows, int64_t cols, int64_t ld,
                                                           uint8_t *__restrict__ elems, float *__restrict__ scales, int64_t n_cb)
{
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, LPR = BLOCK128 / EPL, RPP = 256 / LPR, NP = BLOCK128 / RPP;
    fp8_saturate_mode();
    __shared__ uint32_t slot[2][4];
    const int64_t tr = blockIdx.x / n_cb, tc = blockIdx.x - tr * n_cb;
    const int lr = threadIdx.x / LPR, lc = threadIdx.x % LPR;
    const int64_t col = tc * BLOCK128 + lc * EPL, left = cols - col;
    const int n = left >= EPL ? EPL : left > 0 ? (int)left : 0;
    uint4 t[NP];
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int64_t r = tr * BLOCK128 + p * RPP + lr;
        t[p] = load16<DT>(src, r * ld + col, r < rows ? n : 0);
    }
    uint32_t m = group256_max(pieces_max<DT, NP>(t), slot[0]);
    const bool finite = m < 0x7F800000u;
    if (!finite) {                                    // (the whole work-group)
        m = 0;
#pragma unroll 1
        for (int p = 0; p < NP; p++) {
            uint32_t v[EPL];
            widen<DT>(t[0], v);
            const uint32_t k = finite_max(v);
            m = m > k ? m : k;
            const uint4 first = t[0];                 // (the pieces move along: none is indexed by the loop counter)
#pragma unroll
            for (int j = 0; j + 1 < NP; j++) t[j] = t[j + 1];
            t[NP - 1] = first;
        }
        m = group256_max(m, slot[1]);
    }
    const float f = b128_factor<FMT>(m);
    auto put = [&](int p, const uint32_t (&out)[EPL / 4]) {
        const int64_t r = tr * BLOCK128 + p * RPP + lr;
        if (r >= rows) return;
        uint8_t *o = elems + (r * n_cb + tc) * BLOCK128 + lc * EPL;
        if constexpr (EPL == 8) *reinterpret_cast<uint2 *>(o) = make_uint2(out[0], out[1]);
        else *reinterpret_cast<uint32_t *>(o) = out[0];
    };
    if (finite) {
#pragma unroll
        for (int p = 0; p < NP; p++) {
            uint32_t v[EPL], out[EPL / 4];
            widen<DT>(t[p], v);
            b128_convert<FMT, EPL>(v, f, out);
            put(p, out);
        }
    } else {
#pragma unroll 1
        for (int p = 0; p < NP; p++) {
            uint32_t v[EPL], out[EPL / 4];
            widen<DT>(t[0], v);
            b128_convert_any<FMT, EPL>(v, f, out);
            put(p, out);
#pragma unroll
            for (int j = 0; j + 1 < NP; j++) t[j] = t[j + 1];
        }
    }
    if (threadIdx.x == 0) scales[blockIdx.x] = 1.0f / f;
}

// Columns of a work-group: blocks of bf16 are cast in halves of a tile, so that twice as many work-groups fit into the LDS (16384 x 2048 23.0 us, whole
// tiles 24.5; 1000 x 5000 5.6 and 6.6; 8192 x 8192 38.7 and 38.0); Float32 in whole ones (4096 x 8192 34 us, halves 38).
constexpr int cast128_col_width(int dt, bool tile) { return tile || dt != DT_BF16 ? 128 : 64; }

// pieces of 128 rows x W columns of the source, a tile or half of one; piece t = xcd * per_xcd + i: each XCD walks down a run of column strips, so that the
// scales of a column, and the lines of codes that share a page, are written through one L2
template <int FMT, int DT, bool TILE>
__global__ __launch_bounds__(256) void cast128_col_kernel(const void *__restrict__ src, int64_t rows, int64_t cols, int64_t ld,
                                                          uint8_t *__restrict__ elems, float *__restrict__ scales, int64_t n_rb, int64_t n_tiles, int64_t per_xcd)
{
    constexpr int W = cast128_col_width(DT, TILE), EPL = DT == DT_BF16 ? 8 : 4, LPR = W / EPL, RPP = 256 / LPR, NP = BLOCK128 / RPP;
    constexpr int ES = DT == DT_BF16 ? 2 : 4, PITCH = W * ES, TURN = 16 * ES;
    fp8_saturate_mode();
    __shared__ __attribute__((aligned(16))) uint8_t tile[BLOCK128 * PITCH];
    __shared__ uint32_t slot[2][4];
    const int64_t tile_id = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per_xcd || tile_id >= n_tiles) return;   // uniform over the work-group
    const int64_t tc = tile_id / n_rb, tr = tile_id - tc * n_rb;
    {
        const int lr = threadIdx.x / LPR, lc = threadIdx.x % LPR;
        const int64_t col = tc * W + lc * EPL, left = cols - col;
        const int n = left >= EPL ? EPL : left > 0 ? (int)left : 0;
        uint4 t[NP];
#pragma unroll
        for (int p = 0; p < NP; p++) {
            const int64_t r = tr * BLOCK128 + p * RPP + lr;
            t[p] = load16<DT>(src, r * ld + col, r < rows ? n : 0);
        }
#pragma unroll
        for (int p = 0; p < NP; p++) {
            const int r = p * RPP + lr;
            *reinterpret_cast<uint4 *>(tile + r * PITCH + ((lc * 16 + (r >> 5) * TURN) & (PITCH - 1))) = t[p];
        }
    }
    __syncthreads();
    const int rb = threadIdx.x & 3;
    auto column = [&](int c, uint32_t (&v)[32]) {
        const uint8_t *p = tile + rb * 32 * PITCH + ((c * ES + rb * TURN) & (PITCH - 1));
#pragma unroll
        for (int i = 0; i < 32; i++) {
            if constexpr (DT == DT_BF16) v[i] = (uint32_t)*reinterpret_cast<const uint16_t *>(p + i * PITCH) << 16;
            else v[i] = *reinterpret_cast<const uint32_t *>(p + i * PITCH);
        }
    };
    auto store = [&](int64_t col, const uint32_t (&out)[8]) {
        uint8_t *o = elems + (col * n_rb + tr) * BLOCK128 + rb * 32;
        st16(o, make_uint4(out[0], out[1], out[2], out[3]));
        st16(o + 16, make_uint4(out[4], out[5], out[6], out[7]));
    };
    const int c0 = threadIdx.x >> 2;                  // this thread's column (and c0 + 64)
    if constexpr (!TILE) {
#pragma unroll
        for (int h = 0; h < W / 64; h++) {
            const int64_t col = tc * W + c0 + 64 * h;
            uint32_t v[32], out[8];
            column(c0 + 64 * h, v);
            const float f = b128_quantize<FMT, 32>(v, [](uint32_t m) { return group_max<4>(m); }, out);
            if (col < cols) {
                store(col, out);
                if (rb == 0) scales[col * n_rb + tr] = 1.0f / f;
            }
        }
    } else {
        uint32_t v[2][32];
        column(c0, v[0]);
        column(c0 + 64, v[1]);
        uint32_t a = raw_max(v[0]), b = raw_max(v[1]);
        uint32_t m = group256_max(a > b ? a : b, slot[0]);
        const bool finite = m < 0x7F800000u;
        if (!finite) {
            a = finite_max(v[0]); b = finite_max(v[1]);
            m = group256_max(a > b ? a : b, slot[1]);
        }
        const float f = b128_factor<FMT>(m);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int64_t col = tc * BLOCK128 + c0 + 64 * h;
            uint32_t out[8];
            if (finite) b128_convert<FMT, 32>(v[h], f, out);
            else b128_convert_any<FMT, 32>(v[h], f, out);
            if (col < cols) store(col, out);
        }
        if (threadIdx.x == 0) scales[tc * n_rb + tr] = 1.0f / f;
    }
}

template <int FMT, int DT>
static hipError_t launch_cast128_t(const void *src, int64_t rows, int64_t cols, int64_t ld, int axis, bool tile, uint8_t *elems, float *scales, hipStream_t st)
{
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, ES = DT == DT_BF16 ? 2 : 4;
    const int64_t n_rb = (rows + 127) / 128, n_cb = (cols + 127) / 128;
    if (axis == 1 && !tile) {
        // a launch numbers its units with 31 bits: rows in as many launches as that takes
        const int64_t upr = n_cb * (BLOCK128 / EPL), limit = ((int64_t)1 << 31) - 64 * ROW128_CHUNKS * 4;
        if (upr > limit) return hipErrorNotSupported;
        const int64_t most = limit / upr;
        for (int64_t r0 = 0; r0 < rows; r0 += most) {
            const int64_t nr = rows - r0 < most ? rows - r0 : most;
            const Rows128 geom = {fast_div(upr), cols, ld, (uint32_t)(nr * upr)};
            const int64_t per_wg = 64 * ROW128_CHUNKS * 4, grid = (nr * upr + per_wg - 1) / per_wg;
            hipLaunchKernelGGL((cast128_row_kernel<FMT, DT>), dim3((unsigned)grid), dim3(256), 0, st, static_cast<const uint8_t *>(src) + r0 * ld * ES, geom,
                               elems + r0 * n_cb * BLOCK128, scales + r0 * n_cb);
        }
        return hipGetLastError();
    }
    // one work-group a tile, or half of one; the runtime counts a grid's threads in 32 bits
    const int width = axis == 0 ? cast128_col_width(DT, tile) : 128;
    const int64_t n_cs = (cols + width - 1) / width;
    if (n_rb > (((int64_t)1 << 24) - 8) / n_cs) return hipErrorNotSupported;
    const int64_t n_tiles = n_rb * n_cs, per_xcd = (n_tiles + 7) / 8;
    if (axis == 1)
        hipLaunchKernelGGL((cast128_tile_kernel<FMT, DT>), dim3((unsigned)n_tiles), dim3(256), 0, st, src, rows, cols, ld, elems, scales, n_cb);
    else if (tile)
        hipLaunchKernelGGL((cast128_col_kernel<FMT, DT, true>), dim3((unsigned)(per_xcd * 8)), dim3(256), 0, st, src, rows, cols, ld, elems, scales, n_rb, n_tiles, per_xcd);
    else
        hipLaunchKernelGGL((cast128_col_kernel<FMT, DT, false>), dim3((unsigned)(per_xcd * 8)), dim3(256), 0, st, src, rows, cols, ld, elems, scales, n_rb, n_tiles, per_xcd);
    return hipGetLastError();
}

hipError_t launch_cast_b128(const void *src, int src_dt, int64_t rows, int64_t cols, int64_t ld, int axis, bool tile, int fmt, uint8_t *elems, float *scales, hipStream_t st)
{
    if (fmt == FP8_E4M3)
        return src_dt == DT_BF16 ? launch_cast128_t<FP8_E4M3, DT_BF16>(src, rows, cols, ld, axis, tile, elems, scales, st)
                                 : launch_cast128_t<FP8_E4M3, DT_F32>(src, rows, cols, ld, axis, tile, elems, scales, st);
    return src_dt == DT_BF16 ? launch_cast128_t<FP8_E5M2, DT_BF16>(src, rows, cols, ld, axis, tile, elems, scales, st)
                             : launch_cast128_t<FP8_E5M2, DT_F32>(src, rows, cols, ld, axis, tile, elems, scales, st);
}

}  // namespace mx
