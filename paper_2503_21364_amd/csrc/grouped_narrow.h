// What the two kernels over small matrices share: tiles of 16 rows of a wavefront in LDS.
#ifndef LMK_GS_GROUPED_NARROW_H
#define LMK_GS_GROUPED_NARROW_H
#include "grouped_kernels.h"

namespace lmk {

constexpr u32 kTileRows = 16;
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

// A lane's N pieces (four values each) of a tile of rows of `width` >= 4 values.  Where rows end inside a piece, the row's
// last four values are read and moved into place.
template <class T, u32 N> struct Pieces {
    f32x4 next[N];
    u32 from[N], of_row[N];
    bool last[N];
    u32 rest, quads;

    __device__ __forceinline__ void init(u64 ld, u32 width, u32 lane)
    {
        quads = pitch_of(width) / 4;
        rest = width % 4;
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            const u32 piece = lane + i * kWave, m = piece / quads, c = (piece - m * quads) * 4;
            last[i] = c + 4 > width;
            of_row[i] = m < kTileRows && c < width ? m : ~0u;
            from[i] = (m * (u32)ld + (last[i] ? width - 4 : c)) * (u32)sizeof(T);
        }
    }
    // asks for the tile whose first row is p; rows from `rows` on are zeros
    __device__ __forceinline__ void request(const char *p, u32 rows)
    {
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            next[i] = f32x4{};
            if (of_row[i] < rows) next[i] = load4(reinterpret_cast<const T *>(p + from[i]));
        }
    }
    __device__ __forceinline__ void put(float *lds, u32 lane) const
    {
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            f32x4 v = next[i];
            if (rest != 0 && last[i])
                v = rest == 1 ? f32x4{v[3], 0.f, 0.f, 0.f} : rest == 2 ? f32x4{v[2], v[3], 0.f, 0.f} : f32x4{v[1], v[2], v[3], 0.f};
            const u32 piece = lane + i * kWave;
            if (piece < kTileRows * quads) *reinterpret_cast<f32x4 *>(lds + 4 * piece) = v;
        }
    }
};

// A block's weights into LDS, as the matrix instructions take them: step s (four sum indices) of column tile c (16 columns)
// at (s CT + c) 64, a lane's (column, sum index) there.  across: columns contiguous in memory, not sum indices.
template <class T, u32 CT>
__device__ __forceinline__ void stage_weights(float *lw, const T *w, u64 ldw, bool across, u32 sums, u32 cols)
{
    const u32 steps = (sums + 3) / 4;
    if (across) {
        for (u32 i = threadIdx.x; i < steps * 4 * CT * 4; i += 256) {
            const u32 s = i / (CT * 4), c = i % (CT * 4);
            const f32x4 v = s < sums ? load4_of(w + (u64)s * ldw, 4 * c, cols) : f32x4{};
            *reinterpret_cast<f32x4 *>(lw + (s / 4 * CT + c / 4) * kWave + s % 4 * 16 + c % 4 * 4) = v;
        }
    } else {
        for (u32 i = threadIdx.x; i < steps * CT * 16; i += 256) {
            const u32 c = i / steps, s = i % steps;
            const f32x4 v = c < cols ? load4_of(w + (u64)c * ldw, 4 * s, sums) : f32x4{};
#pragma unroll
            for (u32 e = 0; e < 4; ++e) lw[(s * CT + c / 16) * kWave + e * 16 + c % 16] = v[e];
        }
    }
}

}  // namespace lmk
#endif
