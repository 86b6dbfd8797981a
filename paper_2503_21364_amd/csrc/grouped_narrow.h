// What the two kernels over small matrices share: tiles of 16 rows of a wavefront in LDS.
#ifndef LMK_GS_GROUPED_NARROW_H
#define LMK_GS_GROUPED_NARROW_H
#include "grouped_kernels.h"

namespace lmk {

constexpr u32 kTileRows = 16;
// of a compute unit, and how it is given out to workgroups
constexpr u32 kLdsBytes = 160u << 10, kLdsPiece = 1280;
// byte offsets inside a tile are 32 bits wide
constexpr u64 kNarrowStride = 1u << 23;

__device__ __forceinline__ void wave_meets()          // LDS written by other lanes of this wavefront
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Floats between the rows of a tile: 4 (odd), so that the 16 rows and four consecutive columns that an instruction reads are on
// 64 different banks.
__host__ __device__ constexpr u32 pitch_of(u32 width) { return ((width + 3) / 4 | 1) * 4; }

// four values of a row of `width`, from c on; what is beyond it: zeros
template <class T> __device__ __forceinline__ f32x4 load4_of(const T *p, u32 c, u32 width)
{
    if (c + 4 <= width) return load4(p + c);
    f32x4 v = {};
#pragma unroll
    for (u32 e = 0; e < 4; ++e)
        if (c + e < width) v[e] = to_f32(p[c + e]);
    return v;
}

// How a wavefront brings a tile of rows of `width` values, four at a time: as many rows as it has lanes for in a turn, N
// turns.  A lane has the same columns in all of them, so that what it keeps is one offset.
struct Turns {
    u32 row, col;           // of the first turn; row ~0u: a lane without work
    u32 rows;               // of a turn
    u32 to;                 // offset in LDS

    __device__ __forceinline__ void init(u32 width, u32 lane)
    {
        const u32 quads = (width + 3) / 4;
        rows = kWave / quads;
        row = lane / quads;
        col = (lane - row * quads) * 4;
        to = row * pitch_of(width) + col;
        if (row >= rows) row = ~0u;
    }
};
// turns that a tile of at most 4 `quads` values a row takes
__host__ __device__ constexpr u32 turns_of(u32 quads) { return (kTileRows + kWave / quads - 1) / (kWave / quads); }

// Clears what lies between the rows of a tile in LDS, once: no turn writes there.
__device__ __forceinline__ void clear_gaps(float *lds, u32 width, u32 lane)
{
    const u32 pitch = pitch_of(width), from = (width + 3) / 4 * 4, gap = pitch - from;
    if (lane < kTileRows)
        for (u32 c = 0; c < gap; ++c) lds[lane * pitch + from + c] = 0.0f;
}

// Rows of `width` >= 4 values.  Where they end inside four values, the row's last four are read and moved into place.  Rows that
// are not there are read as the first one and put down as zeros: loads under conditions of their own would be waited for
// one after the other.
template <class T, u32 N> struct Pieces {
    Turns t;
    f32x4 next[N];
    u32 first, turn_bytes, turn_floats;
    u32 rest, rows;         // values behind the last whole four; rows of the requested tile
    bool last;              // whether this lane has them

    __device__ __forceinline__ void init(u64 ld, u32 width, u32 lane)
    {
        t.init(width, lane);
        rest = width % 4;
        last = t.col + 4 > width;
        first = (last ? width - 4 : t.col) * (u32)sizeof(T);
        turn_bytes = (u32)ld * (u32)sizeof(T);
        turn_floats = t.rows * pitch_of(width);
    }
    // asks for the tile whose first row is p
    __device__ __forceinline__ void request(const char *p, u32 rows_)
    {
        rows = rows_;
        if (rows == 0) return;
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            const u32 row = t.row + i * t.rows;
            next[i] = load4(reinterpret_cast<const T *>(p + ((t.row < rows && row < rows ? row : 0u) * turn_bytes + first)));
        }
    }
    __device__ __forceinline__ void put(float *lds) const
    {
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            f32x4 v = next[i];
            if (rest != 0) {
                const f32x4 moved = rest == 1 ? f32x4{v[3], 0.f, 0.f, 0.f} : rest == 2 ? f32x4{v[2], v[3], 0.f, 0.f} : f32x4{v[1], v[2], v[3], 0.f};
#pragma unroll
                for (u32 e = 0; e < 4; ++e) v[e] = last ? moved[e] : v[e];
            }
            const u32 row = t.row + i * t.rows;
            if (rows < kTileRows) {
#pragma unroll
                for (u32 e = 0; e < 4; ++e) v[e] = row < rows ? v[e] : 0.0f;
            }
            if (t.row < kTileRows && row < kTileRows) *reinterpret_cast<f32x4 *>(lds + t.to + i * turn_floats) = v;
        }
    }
};

// A block's weights into LDS, as the matrix instructions take them: step s (four sum indices) of column tile c (16 columns)
// at (s CT + c) 64, a lane's (column, sum index) there.  across: columns contiguous in memory, not sum indices.
template <class T, u32 CT>
__device__ __forceinline__ void stage_weights(float *lw, const T *w, u64 ldw, bool across, u32 sums, u32 cols)
{
    // four values of a matrix row of `width` from c on, rows and values that are not there zeros; no load has a condition
    const auto four = [&](u32 row, u32 rows, u32 c, u32 width) {
        const u32 back = c + 4 <= width ? 0u : width >= 4 ? c + 4 - width : 0u;          // the row's last four instead
        const T *p = w + (u64)(row < rows ? row : 0u) * ldw + (c < width ? c - back : 0u);
        f32x4 v;
        if (width >= 4) v = load4(p);
        else
            for (u32 e = 0; e < 4; ++e) v[e] = e < width ? to_f32(p[e]) : 0.0f;
        f32x4 o;
#pragma unroll
        for (u32 e = 0; e < 4; ++e) {
            float f = v[e];
            f = back == 1 ? (e < 3 ? v[e < 3 ? e + 1 : 3] : 0.0f) : f;
            f = back == 2 ? (e < 2 ? v[e < 2 ? e + 2 : 3] : 0.0f) : f;
            f = back == 3 ? (e < 1 ? v[3] : 0.0f) : f;
            o[e] = row < rows && c < width ? f : 0.0f;
        }
        return o;
    };
    const u32 steps = (sums + 3) / 4;
    if (across) {
#pragma unroll 4
        for (u32 i = threadIdx.x; i < steps * 4 * CT * 4; i += 256) {
            const u32 s = i / (CT * 4), c = i % (CT * 4);
            *reinterpret_cast<f32x4 *>(lw + (s / 4 * CT + c / 4) * kWave + s % 4 * 16 + c % 4 * 4) = four(s, sums, 4 * c, cols);
        }
    } else {
#pragma unroll 4
        for (u32 i = threadIdx.x; i < steps * CT * 16; i += 256) {
            const u32 c = i / steps, s = i - c * steps;
            const f32x4 v = four(c, cols, 4 * s, sums);
#pragma unroll
            for (u32 e = 0; e < 4; ++e) lw[(s * CT + c / 16) * kWave + e * 16 + c % 16] = v[e];
        }
    }
}

}  // namespace lmk
#endif
