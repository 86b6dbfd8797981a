// The 4-bit form of 32 values (lmk_gs_block4), and the sizes of its rows.
#ifndef LMK_GS_BLOCK4_H
#define LMK_GS_BLOCK4_H
#include "grouped.h"

namespace lmk {

// bytes of a row of codes (whole steps of the matrix instruction, 128 values) and of scales (16 bytes, 512 values)
__host__ __device__ constexpr u32 code_bytes(u32 k) { return (k + 127) / 128 * 64; }
__host__ __device__ constexpr u32 scale_bytes(u32 k) { return (k + 511) / 512 * 16; }

// scale byte of 32 values from the bits of the largest |x|: the largest is below 7 steps, where it rounds to 6 at most; at most 252 (four steps of
// 2^126 would be infinite)
__device__ __forceinline__ u32 scale4_of_max(u32 top_bits)
{
    u32 s = top_bits >> 23;
    s = s > 2 ? s - 2 : 0u;
    s += (top_bits & 0x7fffffu) >= 0x600000u ? 1u : 0u;
    s = s > 1u ? s : 1u;
    s = s < 252u ? s : 252u;
    s = top_bits >= 0x7f800000u ? 255u : s;
    return top_bits == 0u ? 0u : s;
}
// nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to the even code, and the sign in bit 3.  From 1 on a code is the number's last exponent bits and
// first mantissa bit, below it is the number of halves.
__device__ __forceinline__ u32 code4_of(float v, float inverse)
{
    const float q = __builtin_fabsf(v) * inverse;          // exact: a power of two, unless it is far below 1/2
    const u32 b = __float_as_uint(q);
    const u32 high = ((b + 0x1fffffu + (b >> 22 & 1u)) >> 22) - 252u;
    const u32 low = (u32)__builtin_rintf(q + q);
    const u32 code = q < 1.0f ? low : high;
    return (code < 7u ? code : 7u) | (__float_as_uint(v) >> 28 & 8u);
}
__device__ __forceinline__ float value4_of(u32 code, float step)
{
    const u32 m = code & 7u;
    const float v = m < 2u ? 0.5f * (float)m : __uint_as_float((m + 252u) << 22);
    return __uint_as_float(__float_as_uint(v) | (code & 8u) << 28) * step;
}

}  // namespace lmk
#endif
