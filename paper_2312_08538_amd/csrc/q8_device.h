// 8-bit floating point with a scale for each block of 128: scales, codes and values of eight elements.
#pragma once
#include "layers_device.h"

namespace conef {

// bits of the largest magnitude; a NaN's if there is one (its bits are above infinity's)
__device__ __forceinline__ uint32_t largest(const float v[8])
{
    float m = fabsf(v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __builtin_elementwise_maximum(m, fabsf(v[i]));
    return __float_as_uint(m) & 0x7FFFFFFFu;
}

// the largest over the lanes l ^ 1, l ^ 2 / over l ^ 16, l ^ 32 / over eight or sixteen neighbours
__device__ __forceinline__ uint32_t quad_largest(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t rows_largest(uint32_t m)
{
    auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)r[0], (uint32_t)r[1]);
    r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max((uint32_t)r[0], (uint32_t)r[1]);
}
template <int G>
__device__ __forceinline__ uint32_t neighbours_largest(uint32_t m)
{
    static_assert(G == 8 || G == 16, "");
    m = quad_largest(m);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));
    if constexpr (G == 16) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true));
    return m;
}

// The scale byte of a block whose largest magnitude has these bits: its exponent less that of the format's largest value, one more for a mantissa above
// 1.75 (by a carry), at least 0.
template <bool E5M2>
__device__ __forceinline__ uint32_t q8_scale(uint32_t most)
{
    constexpr uint32_t kHigh = E5M2 ? 15 : 8;
    const uint32_t e = (most + 0x1FFFFFu) >> 23;
    return most >= 255u << 23 ? 255u : max(e, kHigh) - kHigh;
}

// Eight values over the scale of byte `byte` as codes, by the conversion instructions, which take the scale from a float's exponent (0: 2^-127).
template <bool E5M2>
__device__ __forceinline__ uint2 q8_codes(const float v[8], uint32_t byte)
{
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const float scale = __uint_as_float(byte << 23);
    s16x2 lo = {}, hi = {};
    if constexpr (E5M2) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(lo, v[0], v[1], scale, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(lo, v[2], v[3], scale, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(hi, v[4], v[5], scale, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(hi, v[6], v[7], scale, true);
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[0], v[1], scale, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[2], v[3], scale, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[4], v[5], scale, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[6], v[7], scale, true);
    }
    const uint2 c = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    return byte == 255 ? make_uint2(0, 0) : c;
}

// what four codes stand for
template <bool E5M2>
__device__ __forceinline__ void q8_values(uint32_t c, uint32_t byte, float v[4])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float scale = __uint_as_float(byte << 23);
    f32x2 lo, hi;
    if constexpr (E5M2) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(c, scale, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(c, scale, true);
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, true);
    }
    const float nan = __uint_as_float(0x7FC00000u);
    v[0] = byte == 255 ? nan : lo[0];
    v[1] = byte == 255 ? nan : lo[1];
    v[2] = byte == 255 ? nan : hi[0];
    v[3] = byte == 255 ? nan : hi[1];
}

}  // namespace conef
