// Values of 8-bit floating point with a Float32 scale for each block of 128 or each 128 x 128 tile:
// v = fl(code * scale), rounded once more for a bf16 result.  Bound by memory: 1 byte + 4/128 read, 2 or 4 written.
// 8192 x 8192 to bf16 34.9 us (5.8 TB/s), of the transpose's codes 43.9 (4.6); to Float32 54.6 (6.2).
//
//   dequant128_row_kernel   codes in the order of the result.  A lane takes as many codes as make one 16-byte store: 8 (16 lanes a block) or, of a
//       Float32 result, 4; four loads in flight.  (Two 16-byte stores 32 bytes apart leave every line half written: 4.4 TB/s, not 5.9.)
//   dequant128_col_kernel   codes of the transpose.  A work-group brings 64 lines of 128 codes to LDS, 16 bytes a load; a thread then
//       reads 4 x 8 or 4 x 4 codes (dwords, each four codes of one line), transposes them in registers by byte permutes and writes four
//       rows of 16 bytes: 128 or 256 contiguous bytes per row.
#include "mx_b128.hpp"
#include "mx_launch.hpp"

namespace mx {

// 16 bytes of consecutive values of a row of the result, n of them inside it
template <int DT, int N>
__device__ __forceinline__ void store_values(void *__restrict__ dst, int64_t at, int n, const float (&y)[N])
{
    if constexpr (DT == DT_BF16) {
        static_assert(N == 8, "16 bytes");
        uint16_t *o = static_cast<uint16_t *>(dst) + at;
        const uint32_t p[4] = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
        if (n >= 8) {
            st16_nt(o, make_uint4(p[0], p[1], p[2], p[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) o[i] = (uint16_t)(p[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        static_assert(N == 4, "16 bytes");
        float *o = static_cast<float *>(dst) + at;
        if (n >= 4) {
            st16_nt(o, make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])));
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (i < n) o[i] = y[i];
        }
    }
}

constexpr int DEQ128_CHUNKS = 4;

template <int FMT, int DT>
__global__ __launch_bounds__(256) void dequant128_row_kernel(const uint8_t *__restrict__ elems, const float *__restrict__ scales, int tile_shift, int64_t row0,
                                                             FastDiv units_per_row, int64_t cols, int64_t ld, uint32_t n_units, void *__restrict__ dst)
{
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, LPB = BLOCK128 / EPL;      // codes a lane, lanes a block
    const uint32_t u0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * DEQ128_CHUNKS) + (threadIdx.x & 63);
    uint2 d[DEQ128_CHUNKS];
    float s[DEQ128_CHUNKS];
    int64_t at[DEQ128_CHUNKS];
    int n[DEQ128_CHUNKS];
#pragma unroll
    for (int c = 0; c < DEQ128_CHUNKS; c++) {
        const uint32_t u = u0 + c * 64;
        n[c] = 0;
        if (u < n_units) {
            const uint32_t r = units_per_row(u), k = u - r * units_per_row.d;
            const int64_t left = cols - (int64_t)k * EPL;
            n[c] = left >= EPL ? EPL : left > 0 ? (int)left : 0;
            at[c] = (int64_t)r * ld + (int64_t)k * EPL;
            if constexpr (EPL == 8) d[c] = ld8_nt(elems + (int64_t)u * 8);
            else d[c].x = ld4_nt(elems + (int64_t)u * 4);
            s[c] = scales[((row0 + r) >> tile_shift) * (units_per_row.d / LPB) + k / LPB];
        }
    }
#pragma unroll
    for (int c = 0; c < DEQ128_CHUNKS; c++) {
        if (n[c] <= 0) continue;
        const float2 a = fp8_pair<FMT, false>(d[c].x), b = fp8_pair<FMT, true>(d[c].x);
        if constexpr (EPL == 8) {
            const float2 e = fp8_pair<FMT, false>(d[c].y), f = fp8_pair<FMT, true>(d[c].y);
            const float y[8] = {a.x * s[c], a.y * s[c], b.x * s[c], b.y * s[c], e.x * s[c], e.y * s[c], f.x * s[c], f.y * s[c]};
            store_values<DT, 8>(dst, at[c], n[c], y);
        } else {
            const float y[4] = {a.x * s[c], a.y * s[c], b.x * s[c], b.y * s[c]};
            store_values<DT, 4>(dst, at[c], n[c], y);
        }
    }
}

// four dwords of four bytes, transposed
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&o)[4])
{
    const uint32_t p = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), q = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u);
    const uint32_t r = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u), t = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    o[0] = __builtin_amdgcn_perm(q, p, 0x05040100u);
    o[1] = __builtin_amdgcn_perm(q, p, 0x07060302u);
    o[2] = __builtin_amdgcn_perm(t, r, 0x05040100u);
    o[3] = __builtin_amdgcn_perm(t, r, 0x07060302u);
}

template <int FMT, int DT>
__global__ __launch_bounds__(256) void dequant128_col_kernel(const uint8_t *__restrict__ elems, const float *__restrict__ scales, int tile_shift,
                                                             int64_t rows, int64_t cols, int64_t ld, int64_t n_rb, int64_t n_tiles, int64_t per_xcd,
                                                             void *__restrict__ dst)
{
    constexpr int PITCH = BLOCK128 + 4;               // bytes per line: the dword reads below, 4 or 8 lines and consecutive dwords apart, meet 64 banks
    __shared__ __attribute__((aligned(16))) uint8_t tile[64 * PITCH];
    __shared__ float sc[64];
    const int64_t tile_id = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per_xcd || tile_id >= n_tiles) return;   // uniform over the work-group
    const int64_t n_cs = (cols + 63) / 64;
    const int64_t tr = tile_id / n_cs, cs = tile_id - tr * n_cs;               // along the rows of the result first
    const int t = threadIdx.x;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int line = (t >> 3) + 32 * h;
        const int64_t col = cs * 64 + line;
        uint4 d = make_uint4(0, 0, 0, 0);
        if (col < cols) d = ld16_nt(elems + (col * n_rb + tr) * BLOCK128 + (t & 7) * 16);
        uint32_t *o = reinterpret_cast<uint32_t *>(tile + line * PITCH + (t & 7) * 16);
        o[0] = d.x; o[1] = d.y; o[2] = d.z; o[3] = d.w;
    }
    if (t < 64) sc[t] = cs * 64 + t < cols ? scales[((cs * 64 + t) >> tile_shift) * n_rb + tr] : 0.0f;
    __syncthreads();
    constexpr int EPL = DT == DT_BF16 ? 8 : 4, TPR = 64 / EPL, RPP = 256 / TPR * 4;       // columns a thread, threads a row, rows a pass
#pragma unroll
    for (int pass = 0; pass < BLOCK128 / RPP; pass++) {
        const int c0 = (t % TPR) * EPL, r0 = pass * RPP + (t / TPR) * 4;                  // this thread: rows r0 .. r0 + 3, columns c0 .. c0 + EPL - 1
        uint32_t o[EPL / 4][4];
#pragma unroll
        for (int h = 0; h < EPL / 4; h++) {
            uint32_t a[4];
#pragma unroll
            for (int i = 0; i < 4; i++) a[i] = *reinterpret_cast<const uint32_t *>(tile + (c0 + 4 * h + i) * PITCH + r0);
            transpose4(a, o[h]);
        }
        float s[EPL];
#pragma unroll
        for (int i = 0; i < EPL; i++) s[i] = sc[c0 + i];
        const int64_t left = cols - (cs * 64 + c0);
        const int n = left >= EPL ? EPL : left > 0 ? (int)left : 0;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t r = tr * BLOCK128 + r0 + i;
            float y[EPL];
#pragma unroll
            for (int h = 0; h < EPL / 4; h++) {
                const float2 p = fp8_pair<FMT, false>(o[h][i]), q = fp8_pair<FMT, true>(o[h][i]);
                y[4 * h] = p.x * s[4 * h]; y[4 * h + 1] = p.y * s[4 * h + 1]; y[4 * h + 2] = q.x * s[4 * h + 2]; y[4 * h + 3] = q.y * s[4 * h + 3];
            }
            if (r < rows && n > 0) store_values<DT, EPL>(dst, r * ld + cs * 64 + c0, n, y);
        }
    }
}

template <int FMT, int DT>
static hipError_t launch_dequant128_t(const uint8_t *elems, const float *scales, int64_t rows, int64_t cols, int axis, bool tile, void *dst, int64_t ld, hipStream_t st)
{
    constexpr int ES = DT == DT_BF16 ? 2 : 4;
    const int shift = tile ? 7 : 0;
    const int64_t n_rb = (rows + 127) / 128, n_cb = (cols + 127) / 128;
    if (axis == 1) {
        const int64_t per_wg = 64 * DEQ128_CHUNKS * 4, upr = n_cb * (DT == DT_BF16 ? 16 : 32), limit = ((int64_t)1 << 31) - per_wg;
        if (upr > limit) return hipErrorNotSupported;
        const int64_t most = limit / upr;
        for (int64_t r0 = 0; r0 < rows; r0 += most) {
            const int64_t nr = rows - r0 < most ? rows - r0 : most;
            hipLaunchKernelGGL((dequant128_row_kernel<FMT, DT>), dim3((unsigned)((nr * upr + per_wg - 1) / per_wg)), dim3(256), 0, st, elems + r0 * n_cb * BLOCK128, scales,
                               shift, r0, fast_div(upr), cols, ld, (uint32_t)(nr * upr), static_cast<uint8_t *>(dst) + r0 * ld * ES);
        }
        return hipGetLastError();
    }
    const int64_t n_cs = (cols + 63) / 64;
    if (n_rb > (((int64_t)1 << 24) - 8) / n_cs) return hipErrorNotSupported;
    const int64_t n_tiles = n_rb * n_cs, per_xcd = (n_tiles + 7) / 8;
    hipLaunchKernelGGL((dequant128_col_kernel<FMT, DT>), dim3((unsigned)(per_xcd * 8)), dim3(256), 0, st, elems, scales, shift, rows, cols, ld, n_rb, n_tiles, per_xcd, dst);
    return hipGetLastError();
}

hipError_t launch_dequant_b128(const uint8_t *elems, const float *scales, int fmt, int64_t rows, int64_t cols, int axis, bool tile, void *dst, int dst_dt, int64_t ld,
                               hipStream_t st)
{
    if (fmt == FP8_E4M3)
        return dst_dt == DT_BF16 ? launch_dequant128_t<FP8_E4M3, DT_BF16>(elems, scales, rows, cols, axis, tile, dst, ld, st)
                                 : launch_dequant128_t<FP8_E4M3, DT_F32>(elems, scales, rows, cols, axis, tile, dst, ld, st);
    return dst_dt == DT_BF16 ? launch_dequant128_t<FP8_E5M2, DT_BF16>(elems, scales, rows, cols, axis, tile, dst, ld, st)
                             : launch_dequant128_t<FP8_E5M2, DT_F32>(elems, scales, rows, cols, axis, tile, dst, ld, st);
}

}  // namespace mx
