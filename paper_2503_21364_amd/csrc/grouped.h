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

// Values moved down by d places, zeros behind them; as many places as there are and more: zeros
__device__ __forceinline__ f32x4 moved(f32x4 v, u32 d)
{
    if (d == 0) return v;
    return f32x4{d == 1 ? v[1] : d == 2 ? v[2] : d == 3 ? v[3] : 0.0f, d == 1 ? v[2] : d == 2 ? v[3] : 0.0f, d == 1 ? v[3] : 0.0f, 0.0f};
}
__device__ __forceinline__ bf16x4 moved(bf16x4 v, u32 d)
{
    return __builtin_bit_cast(bf16x4, d < 4 ? __builtin_bit_cast(u64, v) >> (16 * d) : (u64)0);
}
__device__ __forceinline__ bf16x8 moved(bf16x8 v, u32 d)
{
    typedef __attribute__((ext_vector_type(2))) u64 u64x2;
    const u64x2 b = __builtin_bit_cast(u64x2, v);
    u64 lo = b[0], hi = b[1];
    if (d >= 8) {
        lo = hi = 0;
    } else if (d >= 4) {
        lo = hi >> (16 * (d - 4));
        hi = 0;
    } else if (d > 0) {
        lo = lo >> (16 * d) | hi << (64 - 16 * d);
        hi >>= 16 * d;
    }
    return __builtin_bit_cast(bf16x8, u64x2{lo, hi});
}

// The rows a workgroup works on: run `local` of `per` rows of the rows begin..end of a block.
struct RowRun {
    u32 block, begin, end, local;            // block == ~0u: rows of no block
    bool found;
};

// Run number `t` when the runs of all blocks are counted through, in order.  Every block's rows are cut
// into runs of `per` rows by themselves, so the boundaries of the blocks are the only thing a workgroup has to
// look up; 64 blocks are looked at in a step (their run counts, a sum over the lanes, the lane that t falls
// to).  The rows in front of the first block and behind the last one count as blocks too.  Offsets are bounded by `rows`
// whatever they hold, so no run leaves the arrays.  All lanes of a wavefront take part; the result is uniform.
__device__ __forceinline__ RowRun find_run(const u32 *__restrict__ offsets, u32 blocks, u32 rows, u32 per, u32 t)
{
    const u32 lane = threadIdx.x & (kWave - 1);
    const u32 segments = blocks + 2;
    const auto edge = [&](u32 s, u32 &b, u32 &e) {           // rows of segment s; only requests
        b = e = 0;
        if (s >= segments) return;
        b = s == 0 ? 0u : offsets[s - 1];
        e = s == blocks + 1 ? rows : offsets[s];
    };
    u32 before = 0, next_b, next_e;
    edge(lane, next_b, next_e);
    for (u32 base = 0; base < segments; base += kWave) {
        u32 b = next_b, e = next_e;
        edge(base + kWave + lane, next_b, next_e);
        b = b < rows ? b : rows;
        e = e < rows ? e : rows;
        e = e > b ? e : b;
        const u32 count = (e - b + per - 1) / per;
        const u32 upto = before + wave_scan(count);
        const u64 past = __builtin_amdgcn_ballot_w64(upto > t);
        if (past != 0ull) {
            const int at = __builtin_ctzll(past);
            RowRun r;
            r.begin = (u32)__builtin_amdgcn_readlane((int)b, at);
            r.end = (u32)__builtin_amdgcn_readlane((int)e, at);
            r.local = t - ((u32)__builtin_amdgcn_readlane((int)upto, at) - (u32)__builtin_amdgcn_readlane((int)count, at));
            const u32 seg = base + (u32)at;
            r.block = seg == 0 || seg == blocks + 1 ? ~0u : seg - 1;
            r.found = true;
            return r;
        }
        before = wave_last(upto);
    }
    RowRun none = {};
    none.found = false;
    return none;
}

// what is the same in all lanes, in scalar registers
__device__ __forceinline__ u32 uniform(u32 v) { return (u32)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ u64 uniform64(u64 v) { return (u64)uniform((u32)(v >> 32)) << 32 | uniform((u32)v); }

// The same value, of which the compiler knows nothing: what is computed from it inside a loop is not kept in registers across it.
__device__ __forceinline__ u32 afresh(u32 v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// ---- sums over the rows of blocks, in two arrangements.
// By slices: the rows of all blocks are cut into slices of `per` rows, whatever the blocks' lengths are, and the workgroups of a
// slice sum it block after block; a run is where a slice and a block meet.  Every workgroup has the same number of rows.
// By blocks: every block is cut into as many runs of at most `per` rows as it takes, of equal length; a workgroup has one run.
// A block of one run has its result there, one without rows gets its zeros from join_kernel.  Otherwise run r of block g is set r + g + (first row of g) / per of the partial sums,
// rows counted from the first block's; no two runs have the same, in either arrangement (a block's rows / per, rounded up, is at
// most one more than what the first row of the next one adds), and join_kernel adds a block's sets in their order.
struct RowSlices {
    const u32 *offsets;
    u32 blocks, rows, per;      // per: rows of a slice
    u32 front, back;            // first row of the first block, end of the last one

    __device__ __forceinline__ void init(const u32 *offsets_, u32 blocks_, u32 rows_, u32 per_)
    {
        offsets = offsets_;
        blocks = blocks_;
        rows = rows_;
        per = per_;
        front = offsets[0] < rows ? offsets[0] : rows;
        back = offsets[blocks] < rows ? offsets[blocks] : rows;
        back = back > front ? back : front;
    }
    __device__ __forceinline__ void block(u32 g, u32 &b, u32 &e) const
    {
        b = offsets[g] < rows ? offsets[g] : rows;
        e = offsets[g + 1] < rows ? offsets[g + 1] : rows;
        e = e > b ? e : b;
    }
    __device__ __forceinline__ u32 edge(u32 s) const { return back - front > s * per ? front + s * per : back; }
    __device__ __forceinline__ u32 slice_of(u32 row) const { return row > front ? (row - front) / per : 0u; }
};

// The runs of slice s, one after the other; all lanes of a wavefront take part, the results are uniform.
struct SliceRuns {
    RowSlices all;
    u32 s, s0, s1, g;
    u32 block, row, count;      // of the present run
    bool whole;                 // the block has no other

    __device__ __forceinline__ void init(const u32 *offsets, u32 blocks, u32 rows, u32 per, u32 s_)
    {
        all.init(offsets, blocks, rows, per);
        s = s_;
        all.front = uniform(all.front);
        all.back = uniform(all.back);
        s0 = all.edge(s);
        s1 = all.edge(s + 1);
        g = 0;
    }
    // 64 blocks are looked at in a step
    __device__ __forceinline__ bool next()
    {
        const u32 lane = threadIdx.x & (kWave - 1);
        for (; g < all.blocks; g += kWave) {
            u32 b = 0, e = 0;
            if (g + lane < all.blocks) all.block(g + lane, b, e);
            const u64 hit = __builtin_amdgcn_ballot_w64(e > s0 && e > b);
            if (hit == 0ull) continue;
            const int at = __builtin_ctzll(hit);
            b = (u32)__builtin_amdgcn_readlane((int)b, at);
            e = (u32)__builtin_amdgcn_readlane((int)e, at);
            if (b >= s1) return false;
            row = b > s0 ? b : s0;
            count = (e < s1 ? e : s1) - row;
            whole = b >= s0 && e <= s1;
            block = g + (u32)at;
            g = block + 1;
            return true;
        }
        return false;
    }
    __device__ __forceinline__ u32 partial() const { return s + block; }
};

// Run `t` (number of its set) by blocks: looked up by 64 blocks at a time.
struct BlockRun {
    u32 block, row, count, set;
    bool whole;

    __device__ __forceinline__ bool find(const u32 *offsets, u32 blocks, u32 rows, u32 per, u32 t)
    {
        RowSlices all;
        all.init(offsets, blocks, rows, per);
        const u32 lane = threadIdx.x & (kWave - 1);
        for (u32 base = 0; base < blocks; base += kWave) {
            const u32 g = base + lane;
            u32 b = 0, e = 0, first = ~0u, runs = 0;
            if (g < blocks) {
                all.block(g, b, e);
                runs = (e - b + per - 1) / per;
                first = g + all.slice_of(b);
            }
            const u64 hit = __builtin_amdgcn_ballot_w64(first <= t && t - first < runs);
            if (hit == 0ull) continue;
            const int at = __builtin_ctzll(hit);
            const u32 begin = (u32)__builtin_amdgcn_readlane((int)b, at), length = (u32)__builtin_amdgcn_readlane((int)e, at) - begin;
            const u32 n = (u32)__builtin_amdgcn_readlane((int)runs, at), r = t - (u32)__builtin_amdgcn_readlane((int)first, at);
            // equal lengths: the first `longer` runs have one row more
            const u32 share = length / n, longer = length - share * n;
            block = base + (u32)at;
            row = begin + r * share + (r < longer ? r : longer);
            count = share + (r < longer ? 1u : 0u);
            whole = n == 1;
            set = t;
            return true;
        }
        return false;
    }
    __device__ __forceinline__ u32 partial() const { return set; }
};

// Number of slices (host) for tiles that `pairs` workgroups a slice sum, `slots` of them at once: the least of what the last turn's
// workgroups take, with a run's own costs, and what a set of partial sums more costs, its bytes written and read.  A run's own costs (its
// first loads, its results) are more than those of 64 rows: slices are not made shorter for their rows' sake, but for their
// blocks' (64 rows in 64 blocks of 256 x 512, bfloat16, in slices of 64 rows: 486 us, of one row: 30).
struct Slices {
    u32 count;
    double us;              // expected
};
inline Slices slices_of(u32 rows, u32 blocks, u64 pairs, u32 slots, double row_us, double run_us, u64 sums)
{
    const double set_us = (double)sums * 8 / 4e6;
    const u64 most = (u64)rows / 64 + (rows < blocks ? rows : blocks);
    u32 best = 1;
    double least = -1;
    const auto look = [&](u64 n) {
        n = n < most ? n : most;
        if (n == 0) return;
        const double turns = (double)((n * pairs + slots - 1) / slots);
        const double us = turns * ((double)rows / (double)n * row_us + (double)(blocks + n - 1) / (double)n * run_us) + (double)(n - 1) * set_us;
        if (least < 0 || us < least) {
            least = us;
            best = (u32)n;
        }
    };
    for (u64 n = 1; n < 4096; n *= 2) look(n);
    for (u32 turns = 1; turns <= 4; ++turns) look((u64)turns * slots / pairs);
    return Slices{best, least};
}
// rows of each of `slices` slices: s * per stays below 2^32
inline u32 rows_of_slice(u32 rows, u32 slices)
{
    const u32 per = (u32)(((u64)rows + slices - 1) / slices);
    return per < 1 ? 1 : per;
}

// Upper bound of the number of runs (host): every block can end with a run that is not full.
inline u64 max_runs(u32 rows, u32 blocks, u32 per)
{
    const u64 all = (u64)(rows / per) + blocks + 2;
    return all < rows ? all : rows;
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
