// The 8-bit form of activations (include/checkpoint8.h) as its kernels and norm_rotate's share it: a byte for the
// power of two of a group, a signed byte for each value.
#pragma once

#include "common.h"

namespace trimul {

// The power's byte from the bits of the largest magnitude.  64 m rounds to more than 127 from m = 127.5 / 64 on, a
// mantissa of 0x7f0000 (the tie rounds to the even 128); a biased exponent E gives k + 127 = E - 6 or E - 5, at most 248.
__device__ __forceinline__ uint32_t power_byte(uint32_t amax_bits) {
    const uint32_t E = amax_bits >> 23, b = E + ((amax_bits & 0x7fffffu) >= 0x7f0000u ? 1u : 0u);
    return E == 255 ? 255u : b < 6 ? 0u : min(b - 6, 248u);
}
// Whether codes of this group reach 128, which k = 121 has to cut off (127 2^121 is kTopValue).
__device__ __forceinline__ bool power_cut(uint32_t amax_bits) { return amax_bits >= 0x7f7f0000u; }
constexpr float kTopValue = 0x1.fcp127f;
// 2^-k, a normal number for every byte but 255 (of which no code is looked at).
__device__ __forceinline__ float power_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }
// 2^k (2^-127 is subnormal), NaN for 255.
__device__ __forceinline__ float power_value(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}

// Four codes: x 2^-k is exact, and adding 1.5 2^23 rounds it to a whole number, whose low byte is the code.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inverse) {
    constexpr float kWhole = 12582912.f;
    const uint32_t ua = __float_as_uint(__builtin_fmaf(a, inverse, kWhole)), ub = __float_as_uint(__builtin_fmaf(b, inverse, kWhole));
    const uint32_t uc = __float_as_uint(__builtin_fmaf(c, inverse, kWhole)), ud = __float_as_uint(__builtin_fmaf(d, inverse, kWhole));
    const uint32_t lo = __builtin_amdgcn_perm(ub, ua, 0x0c0c0400u), hi = __builtin_amdgcn_perm(ud, uc, 0x04000c0cu);
    return lo | hi;
}
// Code i (0..3) of a word, as a float.
__device__ __forceinline__ float code_value(uint32_t w, int i) { return (float)(int)(int8_t)(w >> (8 * i)); }

// The largest of G consecutive lanes (a power of two up to 32), in all of them.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, false));
}
template <int G>
__device__ __forceinline__ uint32_t umax_lanes(uint32_t v) {
    if constexpr (G >= 2) v = dpp_umax<0xb1>(v);     // quad_perm [1, 0, 3, 2]
    if constexpr (G >= 4) v = dpp_umax<0x4e>(v);     // quad_perm [2, 3, 0, 1]
    if constexpr (G >= 8) v = dpp_umax<0x141>(v);    // row_half_mirror
    if constexpr (G >= 16) v = dpp_umax<0x140>(v);   // row_mirror
    if constexpr (G >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    return v;
}

}  // namespace trimul
