// What the grouped layers' kernels share: which rows a workgroup has, the two element types, and the
// 8-bit form of 32 values.
#ifndef LMK_GS_GROUPED_H
#define LMK_GS_GROUPED_H
#include "lmk_gs_internal.h"
#include "wave_ops.h"

namespace lmk {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// Vectors at any address their elements may have: the rows of the matrices here start where they will, and the
// vector memory instructions take that.
template <class V, class T> __device__ __forceinline__ V load_any(const T *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V, class T> __device__ __forceinline__ void store_any(T *p, V v) { __builtin_memcpy(p, &v, sizeof(V)); }

__device__ __forceinline__ f32x4 load4(const float *p) { return load_any<f32x4>(p); }
__device__ __forceinline__ f32x4 load4(const __bf16 *p)
{
    const bf16x4 v = load_any<bf16x4>(p);
    return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
__device__ __forceinline__ void store4(float *p, f32x4 v) { store_any(p, v); }
__device__ __forceinline__ void store4(__bf16 *p, f32x4 v)
{
    store_any(p, bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]});
}

// The rows a workgroup works on: run `local` of `per` rows of the rows begin..end of a block.
struct RowRun {
    u32 block, begin, end, local, runs;      // block == ~0u: rows of no block
    bool found;
};

// Run number `t` when the runs of all blocks are counted through, in order.  Every block's rows are cut
// into runs of `per` rows by themselves, so the boundaries of the blocks are the only thing a workgroup has to
// look up; 64 blocks are looked at in a step (their run counts, a sum over the lanes, the lane that t falls
// to).  OUTSIDE: the rows in front of the first block and behind the last one count as blocks too, and a block
// without rows has no run; otherwise it has one, and rows of no block have none.  Offsets are bounded by `rows`
// whatever they hold, so no run leaves the arrays.  All lanes of a wavefront take part; the result is uniform.
template <bool OUTSIDE>
__device__ __forceinline__ RowRun find_run(const u32 *__restrict__ offsets, u32 blocks, u32 rows, u32 per, u32 t)
{
    const u32 lane = threadIdx.x & (kWave - 1);
    const u32 segments = OUTSIDE ? blocks + 2 : blocks;
    const auto edge = [&](u32 s, u32 &b, u32 &e) {           // rows of segment s; only requests
        b = e = 0;
        if (s >= segments) return;
        if (OUTSIDE) {
            b = s == 0 ? 0u : offsets[s - 1];
            e = s == blocks + 1 ? rows : offsets[s];
        } else {
            b = offsets[s];
            e = offsets[s + 1];
        }
    };
    u32 before = 0, next_b, next_e;
    edge(lane, next_b, next_e);
    for (u32 base = 0; base < segments; base += kWave) {
        u32 b = next_b, e = next_e;
        edge(base + kWave + lane, next_b, next_e);
        b = b < rows ? b : rows;
        e = e < rows ? e : rows;
        e = e > b ? e : b;
        u32 count = (e - b + per - 1) / per;
        if (!OUTSIDE && count == 0 && base + lane < segments) count = 1;
        const u32 upto = before + wave_scan(count);
        const u64 past = __builtin_amdgcn_ballot_w64(upto > t);
        if (past != 0ull) {
            const int at = __builtin_ctzll(past);
            RowRun r;
            r.begin = (u32)__builtin_amdgcn_readlane((int)b, at);
            r.end = (u32)__builtin_amdgcn_readlane((int)e, at);
            r.runs = (u32)__builtin_amdgcn_readlane((int)count, at);
            r.local = t - ((u32)__builtin_amdgcn_readlane((int)upto, at) - r.runs);
            const u32 seg = base + (u32)at;
            r.block = !OUTSIDE ? seg : (seg == 0 || seg == blocks + 1 ? ~0u : seg - 1);
            r.found = true;
            return r;
        }
        before = wave_last(upto);
    }
    RowRun none = {};
    none.found = false;
    return none;
}

// First row of run `local` of a block whose rows are shared out evenly over its runs (the sums over rows, whose runs need not
// be full ones); run.runs: the end.
__device__ __forceinline__ u32 run_row(const RowRun &run, u32 local)
{
    return run.begin + (u32)((u64)(run.end - run.begin) * local / run.runs);
}

// Upper bound of the number of runs (host): every block can end with a run that is not full.
inline u64 max_runs(u32 rows, u32 blocks, u32 per, bool outside)
{
    const u64 full = rows / per;
    if (outside) {
        const u64 all = full + blocks + 2;
        return all < rows ? all : rows;
    }
    return full + blocks;
}

// ---- 8 bits: 32 values share a power of two
// scale byte of 32 values from the bits of the largest |x|; exponent field - 6, one more where the largest would
// round to 128, at least 1 and at most 248 (64 * 2^122 would be infinite)
__device__ __forceinline__ u32 scale_of_max(u32 top_bits)
{
    u32 s = top_bits >> 23;
    s = s > 6 ? s - 6 : 0u;
    s += (top_bits & 0x7fffffu) >= 0x7f0000u ? 1u : 0u;
    s = s > 1u ? s : 1u;
    s = s < 248u ? s : 248u;
    s = top_bits >= 0x7f800000u ? 255u : s;
    return top_bits == 0u ? 0u : s;
}
// 1 / step; for the bytes 0 and 255 anything finite: the codes are 0 there
__device__ __forceinline__ float inverse_step(u32 scale)
{
    return __uint_as_float((scale == 0u || scale == 255u) ? 0u : (254u - scale) << 23);
}
// step; 0 for the byte 0, infinity for 255 (0 * infinity: what cannot be held reads back as NaN)
__device__ __forceinline__ float step_of(u32 scale) { return __uint_as_float(scale << 23); }

__device__ __forceinline__ int code_of(float v, float inverse)
{
    // v * inverse is exact (a power of two) unless it is far below 1/2
    int c = (int)rintf(fminf(fmaxf(v * inverse, -127.0f), 127.0f));
    c = (c == 0 && v > 0.0f) ? 1 : c;
    c = (c == 0 && v < 0.0f) ? -1 : c;
    return inverse == 0.0f ? 0 : c;
}
__device__ __forceinline__ u32 pack_codes(int a, int b, int c, int d)
{
    return ((u32)a & 255u) | (((u32)b & 255u) << 8) | (((u32)c & 255u) << 16) | ((u32)d << 24);
}
__device__ __forceinline__ float value_of(u32 codes, u32 i, float step)
{
    return (float)(int)(signed char)(codes >> (8 * i)) * step;
}

}  // namespace lmk
#endif
