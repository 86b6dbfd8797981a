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
// Eight codes of eight values, and the way back: the conversion instructions divide by the step (multiply by it), exactly, and round to the
// nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to the even code, at most to 6; they keep the sign of a zero.
typedef __attribute__((ext_vector_type(8))) float f32x8;
__device__ __forceinline__ u32 codes4_of(f32x8 v, float step)
{
    u32 o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], step, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[2], v[3], step, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[4], v[5], step, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[6], v[7], step, 3);
}
__device__ __forceinline__ u32 codes4_of(bf16x8 v, float step)
{
    u32 o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_shufflevector(v, v, 0, 1), step, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_shufflevector(v, v, 2, 3), step, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_shufflevector(v, v, 4, 5), step, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_shufflevector(v, v, 6, 7), step, 3);
}
__device__ __forceinline__ f32x8 values4_of(u32 codes, float step)
{
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, step, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, step, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, step, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, step, 3);
    return f32x8{a[0], a[1], b[0], b[1], c[0], c[1], e[0], e[1]};
}
// largest magnitude of eight values, as the bits of a float32
__device__ __forceinline__ u32 top_of(f32x8 v)
{
    u32 top = 0;
#pragma unroll
    for (u32 j = 0; j < 8; ++j) {
        const u32 b = __float_as_uint(v[j]) & 0x7fffffffu;
        top = top > b ? top : b;
    }
    return top;
}
__device__ __forceinline__ u32 top_of(bf16x8 v)
{
    typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;
    const u16x8 b = __builtin_elementwise_max(__builtin_bit_cast(u16x8, v) & (unsigned short)0x7fff, u16x8{});
    u32 top = 0;
#pragma unroll
    for (u32 j = 0; j < 8; ++j) top = top > b[j] ? top : b[j];
    return top << 16;
}

}  // namespace lmk
#endif
