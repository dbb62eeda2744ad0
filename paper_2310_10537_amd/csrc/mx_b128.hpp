// 8-bit floating point with one Float32 scale for each block of 128 elements of a line (or each 128 x 128 tile):
// the arithmetic that the cast, the fused norm and the dequantize share.  With amax the largest finite magnitude
// of a block and fmax the format's largest number (448 for E4M3, 57344 for E5M2)
//     factor = min(fl(fmax / amax), 2^126) cut to 16 significant bits,   scale = fl(1 / factor),
//     code   = the element nearest to fl(v * factor), ties to even, a NaN a NaN, an infinity NaN (E4M3) or Inf (E5M2).
// The cut makes v * factor exact in Float32 for a bf16 v (8 x 16 bits): a value half way between two elements is
// recognised as such (without it, of bf16 gradients cast to E5M2 about one element in 10^3 went to the wrong side;
// 7 v / amax is a short binary fraction that often).  It moves a scale by at most 2^-15 of itself, which the
// codes make up for.  Because the factor is cut and not rounded, |v| * factor never exceeds fmax by more than a
// rounding of the quotient, so nothing finite overflows.
#pragma once

#include "mx_convert.hpp"

namespace mx {

constexpr int BLOCK128 = 128;

template <int FMT> __device__ __forceinline__ constexpr float fmt_max() { return FMT == FP8_E4M3 ? 448.0f : 57344.0f; }

// amax: bit pattern of the largest finite magnitude
template <int FMT>
__device__ __forceinline__ float b128_factor(uint32_t amax)
{
    const float q = fminf(fmt_max<FMT>() / __uint_as_float(amax), 0x1p126f);
    return __uint_as_float(__float_as_uint(q) & 0xFFFFFF00u);
}

// Maximum over groups of 16 adjacent lanes (a DPP row), in every lane of the group.
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
    v = group_max<4>(v);
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141 /* row_half_mirror */, 0xF, 0xF, false);
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140 /* row_mirror */, 0xF, 0xF, false);
    return v > o ? v : o;
}
// ... of 32 and of 64 adjacent lanes: the row swaps leave a row's and its neighbour's value in one lane of either result
__device__ __forceinline__ uint32_t row32_max(uint32_t v)
{
    v = row16_max(v);
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = row32_max(v);
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}

// N Float32 values (bit patterns), all finite, times factor -> N codes, four to a dword.  The wave is in fp8_saturate_mode().
template <int FMT, int N>
__device__ __forceinline__ void b128_convert(const uint32_t (&v)[N], float factor, uint32_t *out)
{
#pragma unroll
    for (int j = 0; j < N / 4; j++) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = __uint_as_float(v[4 * j + i]) * factor;
        i16x2_t r = {0, 0};
        if constexpr (FMT == FP8_E4M3) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, p[0], p[1], 1.0f, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, p[2], p[3], 1.0f, true);
        } else {
            r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, p[0], p[1], 1.0f, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, p[2], p[3], 1.0f, true);
        }
        out[j] = __builtin_bit_cast(uint32_t, r);
    }
}
// The same for values that may be infinite or NaN.  (A product below the smallest normal Float32 is zero to the encoder, as it is to the format.)
template <int FMT, int N>
__device__ __forceinline__ void b128_convert_any(const uint32_t (&v)[N], float factor, uint32_t *out)
{
#pragma unroll
    for (int j = 0; j < N / 4; j++) {
        uint32_t d = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) d |= encode_elem<FMT, ROUND_RNE>(__float_as_uint(__uint_as_float(v[4 * j + i]) * factor), 127) << (8 * i);
        out[j] = d;
    }
}

template <int N>
__device__ __forceinline__ uint32_t raw_max(const uint32_t (&v)[N])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const uint32_t a = v[i] & 0x7FFFFFFFu;
        m = m > a ? m : a;
    }
    return m;
}
template <int N>
__device__ __forceinline__ uint32_t finite_max(const uint32_t (&v)[N])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const uint32_t a = amax_key<FP8_E4M3>(v[i]);
        m = m > a ? m : a;
    }
    return m;
}

// A lane's N values of a block whose maximum `group` (a function: a lane's maximum -> its block's) completes -> codes; the factor is returned.
template <int FMT, int N, typename Group>
__device__ __forceinline__ float b128_quantize(const uint32_t (&v)[N], Group group, uint32_t *out)
{
    uint32_t amax = group(raw_max(v));
    if (amax < 0x7F800000u) {
        const float f = b128_factor<FMT>(amax);
        b128_convert<FMT, N>(v, f, out);
        return f;
    }
    amax = group(finite_max(v));                      // (every lane of the block comes here)
    const float f = b128_factor<FMT>(amax);
    b128_convert_any<FMT, N>(v, f, out);
    return f;
}

// two codes -> two Float32 values
template <int FMT, bool HI>
__device__ __forceinline__ float2 fp8_pair(uint32_t d)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 r;
    if constexpr (FMT == FP8_E4M3) r = __builtin_amdgcn_cvt_pk_f32_fp8((int)d, HI);
    else r = __builtin_amdgcn_cvt_pk_f32_bf8((int)d, HI);
    return make_float2(r.x, r.y);
}

// two Float32 values -> packed bf16, ties to even, a NaN a NaN
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

}  // namespace mx
