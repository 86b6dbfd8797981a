// What the kernels that take all gradients of small matrices in one pass share (grouped_narrow_bwd.hip, grouped_gated_narrow.hip): from a
// tile of 16 rows of dy and of x in LDS, the sums over rows in a wavefront's registers, dx, and the joining of a workgroup's sums.
#ifndef LMK_GS_GROUPED_NARROW_BWD_H
#define LMK_GS_GROUPED_NARROW_BWD_H
#include "grouped_narrow.h"

namespace lmk {

constexpr u32 kFillers = 64;            // workgroups for dx of rows of no block

// Steps of dx's product, four outputs each, in whole turns of four.  Those behind the last output have zeros on both sides: a
// weight that is not finite, multiplied by a zero of dy, would be a NaN.
__host__ __device__ constexpr u32 whole_steps(u32 n) { return (n + 15) / 16 * 4; }

// floats between the outputs of the joined sums in LDS
constexpr u32 sums_pitch(u32 ck) { return 16 * ck + 4; }
constexpr u32 sums_floats(u32 cn, u32 ck) { return 16 * cn * sums_pitch(ck) + 16 * cn; }

// LDS of the widest matrices of a shape: weights and the four wavefronts' tiles, then their sums in the same place
constexpr u32 shape_lds(u32 cn, u32 ck)
{
    const u32 before = 4 * cn * ck * kWave + 4 * kTileRows * (pitch_of(16 * cn) + pitch_of(16 * ck)), sums = 4 * sums_floats(cn, ck);
    return (before > sums ? before : sums) * 4;
}
// Workgroups of a compute unit (wavefronts of a SIMD), what the registers of the sums and LDS both leave: three up to twelve tiles
// of sums, whose wavefronts take at most 168 registers, two up to 24.  LDS is given out in pieces of 1280 bytes; 64 x 48 and 96 x 32
// have two workgroups for it, 80 x 64 and 96 x 64 one.
constexpr u32 resident(u32 cn, u32 ck)
{
    const u32 registers = cn * ck <= 12 ? 3 : 2, lds = kLdsBytes / ((shape_lds(cn, ck) + kLdsPiece - 1) / kLdsPiece * kLdsPiece);
    return registers < lds ? registers : lds;
}

// Zeros for dx of the rows in front of the first block and behind the last one, by workgroup `filler` of kFillers
__device__ __forceinline__ void fill_outside(const u32 *offsets, u32 blocks, u32 rows, u32 filler, float *dx, u64 lddx, u32 k)
{
    u32 front = offsets[0], back = offsets[blocks];
    front = front < rows ? front : rows;
    back = back < front ? front : back < rows ? back : rows;
    const u32 count = front + (rows - back);
    for (u32 i = filler; i < count && dx; i += kFillers)
        for (u32 c = threadIdx.x; c < k; c += 256) dx[(u64)(i < front ? i : back + (i - front)) * lddx + c] = 0.0f;
}

// Sums over rows: CN, CK: 16 outputs and 16 inputs each
template <u32 CN, u32 CK> struct NarrowSums {
    f32x4 dw[CK][CN];
    float db[CN];

    // Of a tile; columns that are not there hold what lies behind a row, and reach only results that are not kept.
    __device__ __forceinline__ void add(const float *ly, u32 pn, const float *lx, u32 pk, u32 j, u32 q)
    {
        float fy[2][CN], fx[2][CK];
        auto operands = [&](u32 s, u32 at) {
#pragma unroll
            for (u32 b = 0; b < CN; ++b) fy[at][b] = 16 * b + j < pn ? ly[(4 * s + q) * pn + 16 * b + j] : 0.0f;
#pragma unroll
            for (u32 a = 0; a < CK; ++a) fx[at][a] = 16 * a + j < pk ? lx[(4 * s + q) * pk + 16 * a + j] : 0.0f;
        };
        operands(0, 0);
#pragma unroll
        for (u32 s = 0; s < 4; ++s) {
            if (s < 3) operands(s + 1, (s + 1) & 1);
#pragma unroll
            for (u32 b = 0; b < CN; ++b) db[b] += fy[s & 1][b];
#pragma unroll
            for (u32 a = 0; a < CK; ++a)
#pragma unroll
                for (u32 b = 0; b < CN; ++b) dw[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fx[s & 1][a], fy[s & 1][b], dw[a][b], 0, 0, 0);
        }
    }
    // The four wavefronts' sums meet in LDS, [output][input] and then db each, and are added in their order.  Either of to_w and to_b may be NULL.
    __device__ __forceinline__ void join(float *lds, u32 wave, u32 j, u32 q, u32 n, u32 k, bool in_major, float *to_w, float *to_b)
    {
        constexpr u32 ps = sums_pitch(CK), part = sums_floats(CN, CK);
        __syncthreads();
        float *ls = lds + wave * part, *lb = ls + 16 * CN * ps;
#pragma unroll
        for (u32 b = 0; b < CN; ++b) {
            db[b] += __shfl_xor(db[b], 16, kWave);
            db[b] += __shfl_xor(db[b], 32, kWave);
#pragma unroll
            for (u32 a = 0; a < CK; ++a) *reinterpret_cast<f32x4 *>(ls + (16 * b + j) * ps + 16 * a + 4 * q) = dw[a][b];
            if (q == 0) lb[16 * b + j] = db[b];
        }
        __syncthreads();
        const auto joined = [&](u32 at) { return ((lds[at] + lds[part + at]) + lds[2 * part + at]) + lds[3 * part + at]; };
        if (to_w) {
            const u32 width = in_major ? n : k;
#pragma unroll 4
            for (u32 i = threadIdx.x; i < n * k; i += 256) {
                const u32 outer = i / width, inner = i - outer * width;
                to_w[i] = joined(in_major ? inner * ps + outer : outer * ps + inner);
            }
        }
        if (to_b)
            for (u32 i = threadIdx.x; i < n; i += 256) to_b[i] = joined(16 * CN * ps + i);
    }
};

// dx of a tile: `steps` of four outputs; two steps' operands are on their way from LDS while two are multiplied; behind the last one zeros.
// Behind the last whole turn: what lies there in LDS, and is not multiplied
template <u32 CK>
__device__ __forceinline__ void narrow_dx(f32x4 (&acc)[CK], const float *ly, u32 pn, const float *lw, u32 steps, u32 lane, u32 j, u32 q)
{
    float v[2][2], w[2][2][CK];
    auto fetch = [&](u32 s, u32 at) {
#pragma unroll
        for (u32 e = 0; e < 2; ++e) {
            const float y = ly[j * pn + 4 * (s + e) + q];
            v[at][e] = s + e < steps ? y : 0.0f;
#pragma unroll
            for (u32 c = 0; c < CK; ++c) w[at][e][c] = lw[((s + e) * CK + c) * kWave + lane];
        }
    };
    auto multiply = [&](u32 at) {
#pragma unroll
        for (u32 e = 0; e < 2; ++e)
#pragma unroll
            for (u32 c = 0; c < CK; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[at][e][c], v[at][e], acc[c], 0, 0, 0);
    };
    fetch(0, 0);
    for (u32 s = 0; s < steps; s += 4) {
        fetch(s + 2, 1);
        multiply(0);
        fetch(s + 4, 0);
        multiply(1);
    }
}

// four consecutive values a lane of a row of k
template <u32 CK> __device__ __forceinline__ void store_row(float *out, const f32x4 (&acc)[CK], u32 k, u32 q)
{
#pragma unroll
    for (u32 c = 0; c < CK; ++c) {
        const u32 col = 16 * c + 4 * q;
        if (col + 4 <= k) {
            store4(out + col, acc[c]);
        } else {
#pragma unroll
            for (u32 e = 0; e < 3; ++e)
                if (col + e < k) out[col + e] = acc[c][e];
        }
    }
}

}  // namespace lmk
#endif
