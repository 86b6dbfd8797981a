// Tiles of the kernels that take every size, stride, alignment and type, on the float32 matrix instructions: how operands come from
// memory into LDS, and their product.
//
// Both operands of a tile pass through LDS as [sum index][row or column]: a lane of half `hi` feeds sum
// index t + 16 hi to step t, so the 32 lanes of a half read 32 consecutive floats, and with a pitch of 66
// floats the two halves (16 pitches apart) are on different banks, as are the stores of an operand whose
// sum index is contiguous in memory (eight lanes along it, 8 banks apart; eight rows on the banks between).
#ifndef LMK_GS_GROUPED_TILES_H
#define LMK_GS_GROUPED_TILES_H
#include "grouped_kernels.h"

namespace lmk {

constexpr u32 kStep = 32;                 // sum indices of a staged step
constexpr u32 kThreads = 256;

constexpr u32 pitch_of(u32 width) { return width + 2; }

// ---- operands: how a tile of `W` rows (columns) by kStep sum indices comes from memory.  load() only
// requests; store() puts it into LDS.  Out of range: zeros.

// sum index contiguous in memory: element (m, s) at p[m * ld + s]
template <class T, u32 W> struct Along {
    const T *p;
    u64 ld;
    u32 width, sums;        // valid rows, valid sum indices
    float v[W / 8];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, m = c / 8, s = s0 + c % 8 * 4;
            f32x4 q = {0.f, 0.f, 0.f, 0.f};
            if (m < width) {
                const T *a = p + (u64)m * ld + s;
                if (s + 4 <= sums) q = load4(a);
                else {
#pragma unroll
                    for (u32 j = 0; j < 4; ++j)
                        if (s + j < sums) q[j] = to_f32(a[j]);
                }
            }
#pragma unroll
            for (u32 j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, m = c / 8, s = c % 8 * 4;
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[(s + j) * pitch + m] = v[4 * i + j];
        }
    }
};

// rows (columns) contiguous in memory: element (m, s) at p[s * ld + m]
template <class T, u32 W> struct Across {
    const T *p;
    u64 ld;
    u32 width, sums;
    float v[W / 8];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = s0 + c / (W / 4), m = c % (W / 4) * 4;
            f32x4 q = {0.f, 0.f, 0.f, 0.f};
            if (s < sums && m < width) {
                const T *a = p + (u64)s * ld + m;
                if (m + 4 <= width) q = load4(a);
                else {
#pragma unroll
                    for (u32 j = 0; j < 4; ++j)
                        if (m + j < width) q[j] = to_f32(a[j]);
                }
            }
#pragma unroll
            for (u32 j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = c / (W / 4), m = c % (W / 4) * 4;
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[s * pitch + m + j] = v[4 * i + j];
        }
    }
};

// the same from the 8-bit form: rows of kp codes (all of them there), a scale byte for 32
template <u32 W> struct Across8 {
    const u32 *codes;       // of the tile's first row and column
    const uint8_t *scale;
    u32 kp;                 // codes of a row
    u32 width, sums;        // width: codes to the end of the row
    u32 q[W / 32];
    u32 e[W / 32];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = s0 + c / (W / 4), m = c % (W / 4) * 4;
            const bool there = s < sums && m < width;
            q[i] = there ? codes[((u64)s * kp + m) / 4] : 0u;
            e[i] = there ? scale[(u64)s * (kp / 32) + m / 32] : 0u;
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = c / (W / 4), m = c % (W / 4) * 4;
            const float step = step_of(e[i]);
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[s * pitch + m + j] = value_of(q[i], j, step);
        }
    }
};

// Tiles of 64 x 64 results, 32 x 32 a wavefront: four workgroups a compute unit hide what a step waits for, and the
// operands' way through LDS is no limit at this instruction's rate (128 x 128 tiles, two workgroups: 66 instead of 80 TFLOP/s at
// 65 536 x 256 x 256, 101 instead of 104 at 8192 x 4096 x 4096).
constexpr u32 kTile = 64;

// The product of a tile: acc += A B over `sums`.  `each` is called with the staged A of every step.
template <class A, class B, class Each>
__device__ __forceinline__ void tile_product(A &a, B &b, u32 sums, float *lds, f32x16 &acc, Each &&each)
{
    constexpr u32 pitch = pitch_of(kTile), buffer = 2 * kStep * pitch;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const u32 j = lane & 31, hi = lane / 32, m0 = wave / 2 * 32 + j, n0 = wave % 2 * 32 + j;
    a.load(0);
    b.load(0);
    u32 at = 0;
    for (u32 s0 = 0; s0 < sums; s0 += kStep, at ^= 1) {
        float *la = lds + at * buffer, *lb = la + kStep * pitch;
        a.store(la);
        b.store(lb);
        __syncthreads();                     // the other buffer's readers are past the previous one of these
        if (s0 + kStep < sums) {
            a.load(s0 + kStep);
            b.load(s0 + kStep);
        }
        each(la);
        // steps t and t + 16 in one instruction; the last ones of a short tile hold nothing
        const u32 left = sums - s0;
        auto step = [&](u32 t) {
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(la[(t + 16 * hi) * pitch + m0], lb[(t + 16 * hi) * pitch + n0], acc, 0, 0, 0);
        };
        if (left >= 16) {
#pragma unroll
            for (u32 t = 0; t < 16; ++t) step(t);
        } else {
            for (u32 t = 0; t < left; ++t) step(t);
        }
    }
}

// row of a 32 x 32 result that register v of a lane of half hi holds (its column is lane % 32)
__device__ __forceinline__ u32 row_of(u32 v, u32 hi) { return 8 * (v / 4) + 4 * hi + v % 4; }

}  // namespace lmk
#endif
