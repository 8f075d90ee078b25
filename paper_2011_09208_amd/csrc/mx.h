// Values in 8 and 4 bits with one power-of-two scale for every 32 neighbours along the features (the microscaling formats of the
// Open Compute Project): e4m3 (1 sign, 4 exponent, 3 fraction bits, largest 448) and e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6), scales as
// bytes e that stand for 2^(e - 127), 255 for NaN.
#pragma once
#include "gemm_core.h"

namespace ws {

constexpr int MX_GROUP = 32;

// Lanes 4n .. 4n + 3 exchange within their quad: no LDS.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    const uint32_t a = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);       // lane ^ 1
    v = v > a ? v : a;
    const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);       // lane ^ 2
    return v > b ? v : b;
}

// The scale of a group whose largest magnitude has these fp32 bits: the smallest power of two s with amax <= top * s, top the
// largest value of the type, (1 + TOP_FRACTION / 2^23) * 2^TOP_EXPONENT.  No value then rounds beyond the type's range, so nothing
// saturates.  Comparing magnitudes as integers keeps a NaN the largest; infinity and NaN make the whole group NaN.
template <int TOP_EXPONENT, uint32_t TOP_FRACTION>
__device__ __forceinline__ uint32_t group_scale(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23) - TOP_EXPONENT + ((amax_bits & 0x7fffffu) > TOP_FRACTION ? 1 : 0);
    return amax_bits >= 0x7f800000u ? 255u : (uint32_t)(e < 0 ? 0 : e);
}
constexpr int E4M3_TOP_EXPONENT = 8, E2M1_TOP_EXPONENT = 2;
constexpr uint32_t E4M3_TOP_FRACTION = 0x600000u, E2M1_TOP_FRACTION = 0x400000u;               // 1.75 * 2^8 = 448, 1.5 * 2^2 = 6

// 1 / scale.  A finite group's byte is at most 253, so this is a normal number; a NaN group's values count nothing.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float(byte < 254u ? (254u - byte) << 23 : 0u); }

// Byte i of four scales, for the conversion instructions that apply one.  They look at a float's exponent field alone (checked for all 256
// bytes with sign and fraction bits set: 0 is 2^-127 and 255 NaN, as the format has it), so the neighbours' bits may stay.
__device__ __forceinline__ float scale_of(uint32_t four, int i) { return __uint_as_float(i < 3 ? four << (23 - 8 * i) : four >> 1); }

}  // namespace ws
