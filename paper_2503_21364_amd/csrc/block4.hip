// 4-bit form of a matrix, and back (lmk_gs_block4).  Bound by memory: one pass over the values.  Eight consecutive values a lane, so
// that the four lanes of 32 values find their largest by exchanges inside the wavefront; G lanes have a row (16 and 32 where it is no longer, all 64
// for pieces of longer ones), so that where a wavefront is takes no divisions of its lanes, and rows of a few values leave few lanes idle.
// 65 536 x 2048 in bfloat16: 83 us there (340 MB, 4.1 TB/s; 56 of the same values again and again), 57 back (6.0 TB/s).
#include "block4.h"

namespace lmk {

namespace {

constexpr u32 kItem = 8;                    // values of a lane
constexpr u32 kTurns = 4;                   // rows (pieces) that a wavefront has on their way

template <class T> using Eight = T __attribute__((ext_vector_type(8)));

// What turn t of this wavefront has: a row (of a lane's own group), and the first column of the group's 8 G values
struct Piece {
    u32 row, col;
};
template <u32 G> __device__ __forceinline__ Piece piece_of(u64 wave, u32 t, u32 lane, u32 pieces)
{
    const u64 at = wave * kTurns + t;
    if constexpr (G < 64) {
        return Piece{(u32)(at * (64 / G)) + lane / G, 0u};
    } else {
        const u32 row = (u32)(at / pieces);
        return Piece{row, (u32)(at - (u64)row * pieces) * 512u};
    }
}
__device__ __forceinline__ u64 wave_of() { return uniform64((u64)blockIdx.x * 4 + threadIdx.x / kWave); }

template <class T, u32 G>
__global__ __launch_bounds__(256) void pack4_kernel(const T *__restrict__ x, u64 ldx, u32 rows, u32 k, u32 pieces, u32 *__restrict__ codes,
                                                    u32 *__restrict__ scale)
{
    const u32 lane = threadIdx.x & (kWave - 1), quads = code_bytes(k) / 4, scales = scale_bytes(k) / 4;
    const u64 wave = wave_of();
    Eight<T> v[kTurns];
    Piece at[kTurns];
#pragma unroll
    for (u32 t = 0; t < kTurns; ++t) {
        at[t] = piece_of<G>(wave, t, lane, pieces);
        v[t] = Eight<T>{};
        const u32 c = at[t].col + lane % G * kItem;
        if (at[t].row >= rows || c >= k) continue;
        const T *p = x + (u64)at[t].row * ldx + c;
        if (c + kItem <= k) {
            v[t] = load_any<Eight<T>>(p);
        } else {
#pragma unroll
            for (u32 j = 0; j < kItem - 1; ++j)
                if (c + j < k) v[t][j] = p[j];
        }
    }
#pragma unroll
    for (u32 t = 0; t < kTurns; ++t) {
        u32 top = top_of(v[t]);
        u32 other = wave_dpp<0xB1, 0xf>(0u, top);           // lanes 1 0 3 2
        top = top > other ? top : other;
        other = wave_dpp<0x4E, 0xf>(0u, top);               // lanes 2 3 0 1
        top = top > other ? top : other;
        const u32 s = scale4_of_max(top);
        // the four bytes of 16 lanes
        u32 bytes = s << (lane / 4 % 4 * 8);
        bytes |= wave_dpp<0x141, 0xf>(0u, bytes);           // the other quad of eight lanes
        bytes |= wave_dpp<0x140, 0xf>(0u, bytes);           // the other eight of sixteen
        if (at[t].row >= rows) continue;
        const u32 o = s == 255u ? 0u : codes4_of(v[t], step_of(s == 0u ? 127u : s));
        const u32 item = at[t].col / kItem + lane % G;
        if (item < quads) codes[(u64)at[t].row * quads + item] = o;
        if (lane % 16 == 0) {
            u32 *to = scale + (u64)at[t].row * scales + at[t].col / 128 + lane % G / 16;
            *to = bytes;
            // a row of few values has no lanes for the zeros behind its scales
            if (G < 64 && lane % G == G - 16) {
#pragma unroll
                for (u32 e = 1; e <= 4 - G / 16; ++e) to[e] = 0u;
            }
        }
    }
}

template <class T, u32 G>
__global__ __launch_bounds__(256) void unpack4_kernel(const u32 *__restrict__ codes, const uint8_t *__restrict__ scale, u32 rows, u32 k,
                                                      u32 pieces, T *__restrict__ x, u64 ldx)
{
    const u32 lane = threadIdx.x & (kWave - 1), quads = code_bytes(k) / 4;
    const u64 wave = wave_of();
    u32 q[kTurns], s[kTurns];
    Piece at[kTurns];
#pragma unroll
    for (u32 t = 0; t < kTurns; ++t) {
        at[t] = piece_of<G>(wave, t, lane, pieces);
        q[t] = s[t] = 0u;
        const u32 c = at[t].col + lane % G * kItem;
        if (at[t].row >= rows || c >= k) continue;
        q[t] = codes[(u64)at[t].row * quads + c / kItem];
        s[t] = scale[(u64)at[t].row * scale_bytes(k) + c / 32];
    }
#pragma unroll
    for (u32 t = 0; t < kTurns; ++t) {
        const u32 c = at[t].col + lane % G * kItem;
        if (at[t].row >= rows || c >= k) continue;
        f32x8 v = values4_of(q[t], step_of(s[t] == 0u ? 127u : s[t]));
        if (s[t] == 0u || s[t] == 255u) {
            const float none = __uint_as_float(s[t] == 0u ? 0u : 0x7fc00000u);
#pragma unroll
            for (u32 j = 0; j < kItem; ++j) v[j] = s[t] == 0u ? __builtin_copysignf(none, v[j]) : none;
        }
        T *p = x + (u64)at[t].row * ldx + c;
        if (c + kItem <= k) {
            store_any(p, __builtin_convertvector(v, Eight<T>));
        } else {
#pragma unroll
            for (u32 j = 0; j < kItem - 1; ++j)
                if (c + j < k) p[j] = (T)v[j];
        }
    }
}

// Lanes of a row of k values, and the workgroups of four wavefronts
u32 lanes_of(u32 k) { return k <= 128 ? 16 : k <= 256 ? 32 : 64; }
u32 pieces_of(u32 k) { return (k + 511) / 512; }
u64 workgroups(u32 rows, u32 k)
{
    const u32 g = lanes_of(k);
    const u64 turns = g < 64 ? ((u64)rows + 64 / g - 1) / (64 / g) : (u64)rows * pieces_of(k);
    return (turns + 4 * kTurns - 1) / (4 * kTurns);
}

template <class T, u32 G>
hipError_t form_go(void *x, u64 ldx, u32 rows, u32 k, const lmk_gs_block4 &form, bool back, hipStream_t stream)
{
    const dim3 grid((u32)workgroups(rows, k));
    u32 *codes = reinterpret_cast<u32 *>(form.codes);
    if (back) hipLaunchKernelGGL((unpack4_kernel<T, G>), grid, dim3(256), 0, stream, codes, form.scale, rows, k, pieces_of(k), static_cast<T *>(x), ldx);
    else hipLaunchKernelGGL((pack4_kernel<T, G>), grid, dim3(256), 0, stream, static_cast<const T *>(x), ldx, rows, k, pieces_of(k), codes,
                            reinterpret_cast<u32 *>(form.scale));
    return hipGetLastError();
}
template <class T> hipError_t form_as(void *x, u64 ldx, u32 rows, u32 k, const lmk_gs_block4 &form, bool back, hipStream_t stream)
{
    switch (lanes_of(k)) {
    case 16: return form_go<T, 16>(x, ldx, rows, k, form, back, stream);
    case 32: return form_go<T, 32>(x, ldx, rows, k, form, back, stream);
    default: return form_go<T, 64>(x, ldx, rows, k, form, back, stream);
    }
}

}  // namespace

u64 block4_threads(u32 rows, u32 k) { return workgroups(rows, k) * 256; }

hipError_t launch_block4(void *x, u64 ldx, u32 rows, u32 k, u32 dtype, const lmk_gs_block4 &form, bool back, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    return dtype == LMK_GS_F32 ? form_as<float>(x, ldx, rows, k, form, back, stream) : form_as<__bf16>(x, ldx, rows, k, form, back, stream);
}

}  // namespace lmk
