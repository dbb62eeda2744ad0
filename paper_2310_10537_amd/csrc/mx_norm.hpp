// What the RMS norm kernels share: eight consecutive elements of a row per lane and vector.
#pragma once

#include <type_traits>

#include "mx_b128.hpp"
#include "mx_launch.hpp"

namespace mx {

// How a normalised row is delivered beside its own type: one of the MX formats 0 .. 5 (blocks of 32), 8-bit with a
// Float32 scale per 128, or not cast at all
enum : int { OUT_B128_E4M3 = 6, OUT_B128_E5M2 = 7, OUT_NONE = 8 };
__host__ __device__ constexpr int out_block(int out) { return out == OUT_NONE ? 8 : out >= OUT_B128_E4M3 ? 128 : 32; }

// Elements at .. at + 7 of a row of which n lie inside; the rest reads as zero.  The address of a whole vector is 16-byte aligned.
template <int DT, bool NT_LOAD = true>
__device__ __forceinline__ void load8(const void *p, int64_t at, int n, float (&v)[8])
{
    if constexpr (DT == DT_BF16) {
        const uint16_t *q = static_cast<const uint16_t *>(p) + at;
        if (n >= 8) {
            const uint4 t = NT_LOAD ? ld16_nt(q) : ld16(q);
            const uint32_t d[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int i = 0; i < 4; i++) { v[2 * i] = __uint_as_float(d[i] << 16); v[2 * i + 1] = __uint_as_float(d[i] & 0xFFFF0000u); }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = i < n ? __uint_as_float((uint32_t)q[i] << 16) : 0.0f;
        }
    } else {
        const float *q = static_cast<const float *>(p) + at;
        if (n >= 8) {
            const uint4 a = NT_LOAD ? ld16_nt(q) : ld16(q), b = NT_LOAD ? ld16_nt(q + 4) : ld16(q + 4);
            v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
            v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = i < n ? q[i] : 0.0f;
        }
    }
}

// ... rounded to the row's type and stored
template <int DT>
__device__ __forceinline__ void put8(void *p, int64_t at, int n, const float (&v)[8])
{
    if constexpr (DT == DT_BF16) {
        uint16_t *q = static_cast<uint16_t *>(p) + at;
        const uint32_t d[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if (n >= 8) {
            st16(q, make_uint4(d[0], d[1], d[2], d[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) q[i] = (uint16_t)(d[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        float *q = static_cast<float *>(p) + at;
        if (n >= 8) {
            st16(q, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
            st16(q + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) q[i] = v[i];
        }
    }
}

// a Float32 value as the row's type holds it
template <int DT>
__device__ __forceinline__ float held(float v) { return DT == DT_BF16 ? __uint_as_float(pack_bf16(v, 0.0f) << 16) : v; }

__device__ __forceinline__ int inside(int64_t left, int n) { return left >= n ? n : left > 0 ? (int)left : 0; }

// The sum over groups of 16 lanes, and over a wave, in every lane (in one order for all of them)
__device__ __forceinline__ float row16_sum(float v)
{
    auto from = [](float x, auto ctrl) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, false)); };
    v += from(v, std::integral_constant<int, 0xB1>());      // quad_perm [1,0,3,2]
    v += from(v, std::integral_constant<int, 0x4E>());      // quad_perm [2,3,0,1]
    v += from(v, std::integral_constant<int, 0x141>());     // row_half_mirror
    return v + from(v, std::integral_constant<int, 0x140>());   // row_mirror
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = row16_sum(v);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// The sum over the threads that share a row, in each of them: a wave, or the work-group by way of LDS (a float for each of its waves, 16 at most).
template <bool WAVE>
__device__ __forceinline__ float row_sum(float v, float *lds)
{
    v = wave_sum(v);
    if constexpr (!WAVE) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        const int i = threadIdx.x & 15;
        v = row16_sum(i < (int)blockDim.x >> 6 ? lds[i] : 0.0f);
    }
    return v;
}

// Eight codes of an MX block that four adjacent lanes hold -> its scale byte and the lane's codes (8 bit: two dwords, 4 bit: one, 6 bit: 48 bits in two).
// The same codes as the cast of the same Float32 values.
template <int FMT>
__device__ __forceinline__ uint32_t mx_quantize8(const uint32_t (&v)[8], int rnd, uint32_t (&out)[2])
{
    constexpr int w = Fmt<FMT>::bits;
    uint32_t raw = group_max<4>(raw_max(v));
    uint32_t amax = raw;
    if (Fmt<FMT>::elem_nan && raw >= 0x7F800000u) amax = group_max<4>(finite_max(v));     // (all four lanes)
    const uint32_t s = scale_byte<FMT>(amax);
    out[0] = out[1] = 0;
    if (w != 6 && rnd != ROUND_TOWARD_ZERO && raw < 0x7F800000u && (s >= FAST_MIN_SCALE || raw == 0)) {
        const uint32_t fs = fast_scale(s), up = rnd == ROUND_HALF_AWAY ? 1u : 0u;       // (a tie becomes just above the tie)
        const float sf = __uint_as_float(fs << 23);
        auto f = [&](int i) { return __uint_as_float(v[i] | up); };
        if constexpr (w == 8 && FMT != INT8) {
#pragma unroll
            for (int j = 0; j < 2; j++) {
                i16x2_t r = {0, 0};
                if constexpr (FMT == FP8_E4M3) {
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f(4 * j), f(4 * j + 1), sf, false);
                    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f(4 * j + 2), f(4 * j + 3), sf, true);
                } else {
                    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, f(4 * j), f(4 * j + 1), sf, false);
                    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, f(4 * j + 2), f(4 * j + 3), sf, true);
                }
                out[j] = __builtin_bit_cast(uint32_t, r);
            }
        } else if constexpr (FMT == FP4_E2M1) {
            uint32_t q = 0;
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(0), f(1), sf, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(2), f(3), sf, 1);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(4), f(5), sf, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f(6), f(7), sf, 3);
            out[0] = q;
        } else if constexpr (FMT == INT8) {
            // V * 2^(133 - s) is exact; ties away: integer part and fraction apart, ties to even: the magic-number add
            const float c = __uint_as_float((260u - fs) << 23);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float y = __uint_as_float(v[i]) * c;
                if (up) {
                    const float t = truncf(y);
                    y = t + copysignf(fabsf(y - t) >= 0.5f ? 1.0f : 0.0f, y);
                }
                y = __builtin_amdgcn_fmed3f(y, -127.0f, 127.0f);
                out[i >> 2] |= (__float_as_uint(y + 12582912.0f) & 0xFFu) << (8 * (i & 3));
            }
        }
        return s;
    }
    if (!Fmt<FMT>::elem_nan && s == SCALE_NAN) return s;
    // the exact encoder, one element a trip from registers that move along: little code, which counts where a kernel runs for a few microseconds
    // (6 bits: the converts want a whole block in a lane, so this is the only path, and nearest-even is unrolled)
    uint64_t bits = 0;
    if (w == 6 && rnd == ROUND_RNE) {
#pragma unroll
        for (int i = 0; i < 8; i++) bits |= (uint64_t)encode_elem<FMT, ROUND_RNE>(v[i], s) << (w * i);
        out[0] = (uint32_t)bits;
        out[1] = (uint32_t)(bits >> 32);
        return s;
    }
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = v[i];
#pragma unroll 1
    for (int i = 0; i < 8; i++) {
        const uint32_t c = rnd == ROUND_TOWARD_ZERO ? encode_elem<FMT, ROUND_TOWARD_ZERO>(r[0], s)
                           : rnd == ROUND_HALF_AWAY ? encode_elem<FMT, ROUND_HALF_AWAY>(r[0], s) : encode_elem<FMT, ROUND_RNE>(r[0], s);
        bits = (bits >> w) | ((uint64_t)c << (7 * w));
#pragma unroll
        for (int j = 0; j < 7; j++) r[j] = r[j + 1];
    }
    out[0] = (uint32_t)bits;
    out[1] = (uint32_t)(bits >> 32);
    return s;
}

// Vector `vec` (8 elements) of row `row`, which every lane of its block holds a part of, to the row's cast; nvec vectors
// (whole blocks) a row.  All lanes of a wave call it; those without a vector pass on = false.
template <int OUT>
__device__ __forceinline__ void put_cast(const float (&y)[8], int rnd, uint8_t *__restrict__ elems, void *__restrict__ scales, int64_t row, int vec, int nvec, bool on)
{
    if constexpr (OUT != OUT_NONE) {
        uint32_t v[8], out[2];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __float_as_uint(y[i]);
        const int64_t u = row * nvec + vec;
        if constexpr (OUT >= OUT_B128_E4M3) {
            const float f = b128_quantize<OUT == OUT_B128_E4M3 ? FP8_E4M3 : FP8_E5M2, 8>(v, [](uint32_t m) { return row16_max(m); }, out);
            if (on) {
                *reinterpret_cast<uint2 *>(elems + u * 8) = make_uint2(out[0], out[1]);
                if ((vec & 15) == 0) static_cast<float *>(scales)[u >> 4] = 1.0f / f;
            }
        } else {
            constexpr int w = Fmt<OUT>::bits;
            const uint32_t s = mx_quantize8<OUT>(v, rnd, out);
            if constexpr (w == 6) {
                // 24 bytes of four lanes: the even lane of a pair stores the first 8 of their 12 bytes, the odd one the other 4
                const uint32_t o0 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)out[0], 0xB1 /* quad_perm [1,0,3,2] */, 0xF, 0xF, false);
                if (on) {
                    uint32_t *o = reinterpret_cast<uint32_t *>(elems + (u & ~(int64_t)1) * 6);
                    if ((vec & 1) == 0) { o[0] = out[0]; o[1] = out[1] | (o0 << 16); }
                    else o[2] = (out[0] >> 16) | (out[1] << 16);
                }
            } else if (on) {
                if constexpr (w == 8) *reinterpret_cast<uint2 *>(elems + u * 8) = make_uint2(out[0], out[1]);
                else *reinterpret_cast<uint32_t *>(elems + u * 4) = out[0];
            }
            if (on && (vec & 3) == 0) static_cast<uint8_t *>(scales)[u >> 2] = (uint8_t)s;
        }
    }
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    uint8_t *elems;
    void *scales;
    float *rstd;
    int64_t rows, cols, ldx, ldr, ldh, ldy;
    float eps;
    int w_dt, rnd, nvec;
    int64_t row0;         // first row of a launch
};

// rows that one launch may have with `threads` threads for each: the runtime counts a grid's threads in 32 bits
inline int64_t rows_per_launch(int threads) { return (((int64_t)1 << 32) - 1) / threads / 4 * 4; }

}  // namespace mx
