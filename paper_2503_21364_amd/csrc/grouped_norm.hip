// Layer norm of rows whose gain and shift belong to blocks (lmk_gs_grouped_norm), and its gradients.
//     m = mean(x), s = 1 / sqrt(mean((x - m)^2) + eps), h = (x - m) s
//     y = gain_g h + shift_g
//     d = dy gain_g,  dx = s (d - mean(d) - h mean(d h)),  dgain_g = sum of dy h,  dshift_g = sum of dy  over the block's rows
// Everything between the loads and the one rounding of y and dx is in 32 bits.  The squares are of x less the mean, not
// mean(x^2) - m^2: rows far from zero keep their digits.
//
// The mean is a quotient.  In float32 it is rounded, and so are the sums it is taken from: d = x - m is exact where x is far from zero, and what is
// left of a mean in d is summed beside its squares and taken out of both, so that a row of any level has the digits of one of level zero, and a
// row of one value gives its shift.  In bfloat16 sums of values that are alike are exact.
//
// Finite rows have finite statistics: sums are of 2^-16 of the values, of which there are no more than 2^16, d is of their halves, and where its
// squares pass 2^128 all the same, of 2^-80.
//
// Bound by memory: a row is read once.  It stays in the registers of G lanes, C vectors of 16 bytes each, and what is summed
// over it goes from lane to lane without LDS (G <= 64), or through LDS once a sum.  A workgroup has a run of rows of one block,
// so that gain and shift are in registers, and so are its sums of dgain and dshift: x and dy are read once for all three gradients.
//
// The same inputs again and again: 65 536 rows of 1024 in 32 blocks, bfloat16, 49 us (5.4 TB/s), all gradients 91 (4.4 TB/s); 300 000 x 96 in 24,
// float32, 38 (6.0 TB/s; 52 with other inputs every time); 4744 x 4033 in 7, bfloat16, 19, gradients 44: there are four rows a workgroup, and a
// row's two meetings stand behind its loads; one row of 1024 3.0, a chain of latencies.  Sums leave as vectors: with 4 bytes a lane those gradients
// took 55.
#include "grouped_kernels.h"

namespace lmk {

namespace {

struct NormArgs {
    const void *x;              // [rows][k]
    u64 ldx;
    const void *dy;             // [rows][k], of the gradients
    u64 lddy;
    const float *gain, *shift;  // [blocks][k] or NULL
    const u32 *offsets;
    u32 blocks, rows, k;
    float eps;
    void *out;                  // y, or dx, or NULL
    u64 ldo;
    float *dgain, *dshift;      // [blocks][k], either may be NULL
    float *part;                // sets of partial sums: k of dgain, then k of dshift
    f32x4 *stats;               // rows longer than registers: every row's scale, mean times it, off and rate
    u32 per;                    // rows of a run
};

// h = ((x scale - mean scale) - off) rate
constexpr float kOfSum = 0x1p-16f, kHalf = 0.5f, kFar = 0x1p-80f;
__device__ __forceinline__ float mean_of(float sum, u32 k) { return sum / ((float)k * kOfSum); }
__device__ __forceinline__ bool held(float squares) { return squares < __builtin_inff(); }
// Mean of the squares of d, less the square of d's mean, `off`.  Where that is all there is, a difference of roundings would be left: no
// less than 2^-16 of it, beside which d - off is nothing.
__device__ __forceinline__ float variance(float square, float off)
{
    const float var = __builtin_fmaf(-off, off, square), least = off * off * 0x1p-16f;
    return var < least ? least : var;                       // NaN stays
}
// 1 / deviation of d.  0: a row of one value, and nothing of eps is left at this scale; d is 0, too
__device__ __forceinline__ float rate_of(float var, float eps, float scale)
{
    const float q = var + eps * scale * scale;
    return q == 0.0f ? 0.0f : 1.0f / sqrtf(q);
}
// and of x
__device__ __forceinline__ float rate_of_row(float rate, float eps, float scale) { return rate == 0.0f ? 1.0f / sqrtf(eps) : rate * scale; }

template <class T> constexpr u32 kVec = 16 / sizeof(T);
template <class T> constexpr bool kCentred = sizeof(T) == 4;           // off is taken
template <class T> using Vec = T __attribute__((ext_vector_type(16 / sizeof(T))));

// Sum over the G lanes of a row, the same bits in all of them: neighbours, pairs, quads and halves of 16 lanes, then rows of 16 and
// halves of the wavefront exchanged.
template <int CTRL> __device__ __forceinline__ float add_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <u32 G> __device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(G == 8 || G == 16 || G == 64, "lanes of a row");
    typedef __attribute__((ext_vector_type(2))) u32 two;
    v = add_dpp<0xB1>(v);               // quad_perm 1 0 3 2
    v = add_dpp<0x4E>(v);               // quad_perm 2 3 0 1
    v = add_dpp<0x141>(v);              // row_half_mirror
    if constexpr (G >= 16) v = add_dpp<0x140>(v);       // row_mirror
    if constexpr (G == 64) {
        two p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// N sums over the G threads of a row at once.  Rows of several wavefronts meet in LDS; `turn` flips between two places, so that one
// meeting a call is enough: whoever writes a place again has passed the next meeting, and so has everyone who read it.
template <u32 G, u32 N> struct RowSums {
    static constexpr u32 kWaves = G / kWave;
    __device__ __forceinline__ static void of(float (&v)[N], float *lds, u32 &turn)
    {
#pragma unroll
        for (u32 i = 0; i < N; ++i) v[i] = lanes_sum<(G < kWave ? G : kWave)>(v[i]);
        if constexpr (G > kWave) {
            float *at = lds + turn * (kWaves * 4);
            turn ^= 1;
            if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
                for (u32 i = 0; i < N; ++i) at[threadIdx.x / kWave * 4 + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (u32 i = 0; i < N; ++i) {
                if constexpr (kWaves == 16) {           // a wavefront's a lane: sixteen reads would hold 64 registers
                    v[i] = lanes_sum<16>(at[(threadIdx.x & 15) * 4 + i]);
                } else {
                    v[i] = 0.0f;
#pragma unroll
                    for (u32 w = 0; w < kWaves; ++w) v[i] += at[w * 4 + i];
                }
            }
        }
    }
};

// Chunk c of this lane: columns (c G + lane) V and on.  No load has a condition of its own, which would be waited for one after the other: what
// would reach beyond the row is read as its last whole vector, and moved into place when it is used.
template <class T, u32 G, u32 C> struct RowOf {
    static constexpr u32 V = kVec<T>;
    __device__ __forceinline__ static u32 column(u32 c, u32 lane) { return (c * G + lane) * V; }
    // k >= V; rows of fewer are read value by value
    __device__ __forceinline__ static void load(Vec<T> (&v)[C], const T *p, u32 k, u32 lane)
    {
#pragma unroll
        for (u32 c = 0; c < C; ++c) {
            const u32 at = column(c, lane);
            if (k >= V) {
                v[c] = load_any<Vec<T>>(p + (at + V <= k ? at : k - V));
            } else {
#pragma unroll
                for (u32 e = 0; e < V; ++e) v[c][e] = at + e < k ? p[at + e] : (T)0.0f;
            }
        }
    }
    // the values; zeros beyond the row
    __device__ __forceinline__ static void use(float (&f)[C][V], const Vec<T> (&v)[C], u32 k, u32 lane)
    {
#pragma unroll
        for (u32 c = 0; c < C; ++c) {
            const u32 at = column(c, lane);
            Vec<T> w = v[c];
            if (k % V == 0) {
#pragma unroll
                for (u32 e = 0; e < V; ++e) f[c][e] = at < k ? to_f32(w[e]) : 0.0f;
                continue;
            }
            if (k > V) w = moved(w, at + V <= k ? 0u : at - (k - V));
#pragma unroll
            for (u32 e = 0; e < V; ++e) f[c][e] = to_f32(w[e]);
        }
    }
    __device__ __forceinline__ static void store(T *p, const float (&v)[C][V], u32 k, u32 lane)
    {
#pragma unroll
        for (u32 c = 0; c < C; ++c) {
            const u32 at = column(c, lane);
            Vec<T> o;
#pragma unroll
            for (u32 e = 0; e < V; ++e) o[e] = (T)v[c][e];
            if (at + V <= k) {
                store_any(p + at, o);
            } else {
#pragma unroll
                for (u32 e = 0; e < V; ++e)
                    if (at + e < k) p[at + e] = o[e];
            }
        }
    }
    __device__ __forceinline__ static void weights(float (&v)[C][V], const float *p, u32 k, u32 lane, float none)
    {
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 q = 0; q < V; q += 4) {
                const u32 at = column(c, lane) + q;
                f32x4 w = {none, none, none, none};
                if (p && k >= 4) {
                    w = moved(load_any<f32x4>(p + (at + 4 <= k ? at : k - 4)), at + 4 <= k ? 0u : at - (k - 4));
                } else if (p) {
#pragma unroll
                    for (u32 e = 0; e < 4; ++e) w[e] = at + e < k ? p[at + e] : 0.0f;
                }
#pragma unroll
                for (u32 e = 0; e < 4; ++e) v[c][q + e] = w[e];
            }
    }
};

constexpr u32 threads_of(u32 g) { return g > 256 ? g : 256; }

// Rows on their way to a thread of the gradients: two in workgroups of 1024 in bfloat16, of which a compute unit has one (6000 x 8192: 79 us, one row
// 93; in float32 134 and 136)
template <class T, u32 G> constexpr u32 kDeep = G == 1024 && sizeof(T) == 2 ? 2 : 1;
// f(turn, turn % DEEP)
template <u32 DEEP, class F> __device__ __forceinline__ void each_turn(u32 turns, F &&f)
{
    for (u32 t = 0; t < turns; t += DEEP) {
        f(t, std::integral_constant<u32, 0>{});
        if constexpr (DEEP == 2) {
            if (t + 1 < turns) f(t + 1, std::integral_constant<u32, 1>{});
        }
    }
}

template <class T, u32 G, u32 C>
__global__ __launch_bounds__(threads_of(G)) void norm_kernel(const NormArgs r)
{
    using Row = RowOf<T, G, C>;
    constexpr u32 V = Row::V, kAtOnce = threads_of(G) / G;
    __shared__ float meet[2 * 16 * 4];
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, r.per, blockIdx.x);
    if (!run.found) return;
    const u32 lane = threadIdx.x % G, begin = run.begin + run.local * r.per;
    const u32 end = run.end - begin < r.per ? run.end : begin + r.per;
    const bool inside = run.block != ~0u;
    T *out = static_cast<T *>(r.out);
    if (!inside) {
        const float none[C][V] = {};
        for (u32 row = begin + threadIdx.x / G; row < end; row += kAtOnce) Row::store(out + (u64)row * r.ldo, none, r.k, lane);
        return;
    }
    const T *x = static_cast<const T *>(r.x);
    float gain[C][V], shift[C][V];
    const u64 own = (u64)run.block * r.k;
    Row::weights(gain, r.gain ? r.gain + own : nullptr, r.k, lane, 1.0f);
    Row::weights(shift, r.shift ? r.shift + own : nullptr, r.k, lane, 0.0f);
    const float share = 1.0f / (float)r.k;
    u32 turn = 0;
    Vec<T> next[C];
    // threads without a row of their own repeat the run's last one: all meet equally often
    const u32 turns = (end - begin + kAtOnce - 1) / kAtOnce;
    const auto row_at = [&](u32 t) {
        const u32 row = begin + t * kAtOnce + threadIdx.x / G;
        return row < end ? row : end - 1;
    };
    Row::load(next, x + (u64)row_at(0) * r.ldx, r.k, lane);
    for (u32 t = 0; t < turns; ++t) {
        float v[C][V];
        float sum[1] = {0.0f};
        Row::use(v, next, r.k, lane);
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) sum[0] = __builtin_fmaf(v[c][e], kOfSum, sum[0]);
        if (t + 1 < turns) Row::load(next, x + (u64)row_at(t + 1) * r.ldx, r.k, lane);
        RowSums<G, 1>::of(sum, meet, turn);
        const float level = mean_of(sum[0], r.k) * kHalf;
        constexpr u32 kSums = kCentred<T> ? 2 : 1;
        float sums[kSums], scale = kHalf, off = 0.0f;
        const auto square = [&] {
#pragma unroll
            for (u32 i = 0; i < kSums; ++i) sums[i] = 0.0f;
#pragma unroll
            for (u32 c = 0; c < C; ++c)
#pragma unroll
                for (u32 e = 0; e < V; ++e) {
                    sums[0] += v[c][e] * v[c][e];
                    if constexpr (kCentred<T>) sums[1] += v[c][e];
                }
            RowSums<G, kSums>::of(sums, meet, turn);
            if constexpr (kCentred<T>) off = sums[1] * share;
        };
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) v[c][e] = (c * G + lane) * V + e < r.k ? __builtin_fmaf(v[c][e], kHalf, -level) : 0.0f;
        square();
        if (!held(sums[0])) {                       // the same in all threads of the row
#pragma unroll
            for (u32 c = 0; c < C; ++c)
#pragma unroll
                for (u32 e = 0; e < V; ++e) v[c][e] *= kFar / kHalf;
            scale = kFar;
            square();
        }
        const float s = rate_of(variance(sums[0] * share, off), r.eps, scale);
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) v[c][e] = (v[c][e] - off) * s * gain[c][e] + shift[c][e];
        const u32 row = begin + t * kAtOnce + threadIdx.x / G;
        if (row < end) Row::store(out + (u64)row * r.ldo, v, r.k, lane);
    }
}

// Wavefronts of a SIMD that the registers have to leave: three where the compiler would end four registers above (65 536 rows of 1024 in float32, all
// gradients: 171 us, of two 185)
constexpr u32 norm_resident(u32 g, u32 c) { return g == 64 && c == 4 ? 3 : 1; }

// SUMS: dgain and dshift, too
template <class T, u32 G, u32 C, bool SUMS>
__global__ __launch_bounds__(threads_of(G), norm_resident(G, C)) void norm_backward_kernel(const NormArgs r)
{
    using Row = RowOf<T, G, C>;
    constexpr u32 V = Row::V, kThreads = threads_of(G), kAtOnce = kThreads / G;
    __shared__ float meet[2 * 16 * 4];
    __shared__ float copies[SUMS && kAtOnce > 1 ? kThreads * C * V : 1];
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, r.per, blockIdx.x);
    if (!run.found) return;
    const u32 lane = threadIdx.x % G, begin = run.begin + run.local * r.per;
    const u32 end = run.end - begin < r.per ? run.end : begin + r.per;
    const bool inside = run.block != ~0u;
    T *out = static_cast<T *>(r.out);
    if (!inside) {
        const float none[C][V] = {};
        if (out)
            for (u32 row = begin + threadIdx.x / G; row < end; row += kAtOnce) Row::store(out + (u64)row * r.ldo, none, r.k, lane);
        return;
    }
    const T *x = static_cast<const T *>(r.x), *dy = static_cast<const T *>(r.dy);
    float gain[C][V], dgain[C][V] = {}, dshift[C][V] = {};
    const u64 own = (u64)run.block * r.k;
    Row::weights(gain, r.gain ? r.gain + own : nullptr, r.k, lane, 1.0f);
    const float share = 1.0f / (float)r.k;
    u32 turn = 0;
    Vec<T> next_x[kDeep<T, G>][C], next_dy[kDeep<T, G>][C];
    const u32 turns = (end - begin + kAtOnce - 1) / kAtOnce;
    const auto request = [&](u32 t, auto part) {
        u32 row = begin + t * kAtOnce + threadIdx.x / G;
        row = row < end ? row : end - 1;
        Row::load(next_x[part], x + (u64)row * r.ldx, r.k, lane);
        Row::load(next_dy[part], dy + (u64)row * r.lddy, r.k, lane);
    };
#pragma unroll
    for (u32 i = 0; i < kDeep<T, G>; ++i) request(i, i);
    each_turn<kDeep<T, G>>(turns, [&](u32 t, auto part) {
        const u32 row = begin + t * kAtOnce + threadIdx.x / G;
        const bool there = row < end;
        float h[C][V], d[C][V];
        float sum[1] = {0.0f};
        Row::use(h, next_x[part], r.k, lane);
        Row::use(d, next_dy[part], r.k, lane);
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) sum[0] = __builtin_fmaf(h[c][e], kOfSum, sum[0]);
        if (t + kDeep<T, G> < turns) request(t + kDeep<T, G>, part);
        RowSums<G, 1>::of(sum, meet, turn);
        const float mean = mean_of(sum[0], r.k) * kHalf;
        // squares, d, and d (x - m): the last two need no deviation yet
        constexpr u32 kSums = kCentred<T> ? 4 : 3;
        float sums[kSums], scale = kHalf, off = 0.0f;
        const auto square = [&] {
#pragma unroll
            for (u32 i = 0; i < kSums; ++i) sums[i] = 0.0f;
#pragma unroll
            for (u32 c = 0; c < C; ++c)
#pragma unroll
                for (u32 e = 0; e < V; ++e) {
                    const float w = d[c][e] * gain[c][e];
                    sums[0] += h[c][e] * h[c][e];
                    sums[1] += w;
                    sums[2] += w * h[c][e];
                    if constexpr (kCentred<T>) sums[3] += h[c][e];
                }
            RowSums<G, kSums>::of(sums, meet, turn);
            if constexpr (kCentred<T>) off = sums[3] * share;
        };
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) h[c][e] = (c * G + lane) * V + e < r.k ? __builtin_fmaf(h[c][e], kHalf, -mean) : 0.0f;
        square();
        if (!held(sums[0])) {                       // the same in all threads of the row
#pragma unroll
            for (u32 c = 0; c < C; ++c)
#pragma unroll
                for (u32 e = 0; e < V; ++e) h[c][e] *= kFar / kHalf;
            scale = kFar;
            square();
        }
        const float rate = rate_of(variance(sums[0] * share, off), r.eps, scale), s = rate_of_row(rate, r.eps, scale);
        const float level = sums[1] * share, along = (sums[2] * share - off * level) * rate;
#pragma unroll
        for (u32 c = 0; c < C; ++c)
#pragma unroll
            for (u32 e = 0; e < V; ++e) {
                const float g = d[c][e];
                h[c][e] = (h[c][e] - off) * rate;
                if (SUMS && there) {
                    dgain[c][e] += g * h[c][e];
                    dshift[c][e] += g;
                }
                d[c][e] = s * (g * gain[c][e] - level - h[c][e] * along);
            }
        if (there && out) Row::store(out + (u64)row * r.ldo, d, r.k, lane);
    });
    if constexpr (SUMS) {
        const bool alone = run.end - run.begin <= r.per;
        RowSlices all;
        all.init(r.offsets, r.blocks, r.rows, r.per);
        float *set = r.part + (u64)(run.block + all.slice_of(run.begin) + run.local) * 2 * r.k;
        float *to[2] = {alone ? r.dgain ? r.dgain + own : nullptr : set, alone ? r.dshift ? r.dshift + own : nullptr : set + r.k};
#pragma unroll
        for (u32 q = 0; q < 2; ++q) {
            float (&v)[C][V] = q == 0 ? dgain : dshift;
            if constexpr (kAtOnce == 1) {
                if (!to[q]) continue;
#pragma unroll
                for (u32 c = 0; c < C; ++c)
#pragma unroll
                    for (u32 e = 0; e < V; e += 4) {
                        const u32 at = (c * G + lane) * V + e;
                        if (at + 4 <= r.k) {
                            store_any(to[q] + at, f32x4{v[c][e], v[c][e + 1], v[c][e + 2], v[c][e + 3]});
                        } else {
#pragma unroll
                            for (u32 i = 0; i < 3; ++i)
                                if (at + i < r.k) to[q][at + i] = v[c][e + i];
                        }
                    }
            } else {
                // the rows that ran beside each other, added in their order
                constexpr u32 width = G * C * V;
                __syncthreads();
#pragma unroll
                for (u32 c = 0; c < C; ++c)
#pragma unroll
                    for (u32 e = 0; e < V; ++e) copies[threadIdx.x / G * width + (c * G + lane) * V + e] = v[c][e];
                __syncthreads();
                if (!to[q]) continue;
                for (u32 at = threadIdx.x; at < r.k; at += kThreads) {
                    float a = 0.0f;
                    for (u32 w = 0; w < kAtOnce; ++w) a += copies[w * width + at];
                    to[q][at] = a;
                }
            }
        }
    }
}

// ---- rows longer than a workgroup's registers: one row a workgroup of 1024, read again for every pass over it (from cache, mostly)
constexpr u32 kLong = 1024;

// The vectors of a row that this thread has: f(first column, vector that begins there or in front of it, first of its values that counts)
template <class T, class F> __device__ __forceinline__ void each_vector(u32 first, u32 step, u32 k, F &&f)
{
    constexpr u32 V = kVec<T>;
    for (u32 at = first * V; at < k; at += step * V) {
        const u32 from = at + V <= k ? at : k - V;
        f(from, at - from);
    }
}

template <class T, bool BACKWARD>
__global__ __launch_bounds__(kLong) void long_norm_kernel(const NormArgs r)
{
    constexpr u32 V = kVec<T>;
    __shared__ float meet[2 * 16 * 4];
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, 1, blockIdx.x);          // runs of one row
    if (!run.found) return;
    const u32 row = run.begin + run.local;
    const T *x = static_cast<const T *>(r.x) + (u64)row * r.ldx, *dy = static_cast<const T *>(r.dy) + (BACKWARD ? (u64)row * r.lddy : 0);
    T *out = r.out ? static_cast<T *>(r.out) + (u64)row * r.ldo : nullptr;
    if (run.block == ~0u) {
        if (out)
            for (u32 i = threadIdx.x; i < r.k; i += kLong) out[i] = (T)0.0f;
        return;
    }
    const float *gain = r.gain ? r.gain + (u64)run.block * r.k : nullptr, *shift = r.shift ? r.shift + (u64)run.block * r.k : nullptr;
    const float share = 1.0f / (float)r.k;
    u32 turn = 0;
    float sum[1] = {0.0f};
    each_vector<T>(threadIdx.x, kLong, r.k, [&](u32 from, u32 first) {
        const Vec<T> v = load_any<Vec<T>>(x + from);
#pragma unroll
        for (u32 e = 0; e < V; ++e) sum[0] = __builtin_fmaf(e >= first ? to_f32(v[e]) : 0.0f, kOfSum, sum[0]);
    });
    RowSums<kLong, 1>::of(sum, meet, turn);
    const float mean = mean_of(sum[0], r.k);
    float sums[4], scale = kHalf;
    const auto square = [&] {
#pragma unroll
        for (u32 i = 0; i < 4; ++i) sums[i] = 0.0f;
        each_vector<T>(threadIdx.x, kLong, r.k, [&](u32 from, u32 first) {
            const Vec<T> v = load_any<Vec<T>>(x + from);
            Vec<T> g = {};
            if (BACKWARD) g = load_any<Vec<T>>(dy + from);
#pragma unroll
            for (u32 e = 0; e < V; ++e) {
                if (e < first) continue;
                const float h = __builtin_fmaf(to_f32(v[e]), scale, -(mean * scale));
                sums[0] += h * h;
                if (BACKWARD) {
                    const float w = to_f32(g[e]) * (gain ? gain[from + e] : 1.0f);
                    sums[1] += w;
                    sums[2] += w * h;
                }
                if (kCentred<T>) sums[3] += h;
            }
        });
        RowSums<kLong, 4>::of(sums, meet, turn);
    };
    square();
    if (!held(sums[0])) {                           // the same in all threads
        scale = kFar;
        square();
    }
    const float off = sums[3] * share, rate = rate_of(variance(sums[0] * share, off), r.eps, scale), s = rate_of_row(rate, r.eps, scale);
    const float level = sums[1] * share, along = (sums[2] * share - off * level) * rate;
    if (BACKWARD && r.stats && threadIdx.x == 0) r.stats[row] = f32x4{scale, mean * scale, off, rate};
    if (!out) return;
    // out may be x or dy: what a vector holds in front of its first value may have its result already, and is not used
    each_vector<T>(threadIdx.x, kLong, r.k, [&](u32 from, u32 first) {
        const Vec<T> v = load_any<Vec<T>>(x + from);
        Vec<T> g = {}, o;
        if (BACKWARD) g = load_any<Vec<T>>(dy + from);
#pragma unroll
        for (u32 e = 0; e < V; ++e) {
            const float h = (__builtin_fmaf(to_f32(v[e]), scale, -(mean * scale)) - off) * rate, w = gain ? gain[from + e] : 1.0f;
            o[e] = BACKWARD ? (T)(s * (to_f32(g[e]) * w - level - h * along)) : (T)(h * w + (shift ? shift[from + e] : 0.0f));
        }
        if (first == 0) {
            store_any(out + from, o);
        } else {
#pragma unroll
            for (u32 e = 1; e < V; ++e)
                if (e >= first) out[from + e] = o[e];
        }
    });
}

// dgain and dshift of such rows: a thread sums a vector of columns over a run of rows, four of them on their way
template <class T>
__global__ __launch_bounds__(256) void long_norm_sums_kernel(const NormArgs r)
{
    constexpr u32 V = kVec<T>, kRows = 4;
    const u32 pieces = (r.k + 256 * V - 1) / (256 * V), t = blockIdx.x / pieces;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, r.per, t);
    if (!run.found || run.block == ~0u) return;
    const u32 at = ((blockIdx.x - t * pieces) * 256 + threadIdx.x) * V, begin = run.begin + run.local * r.per;
    const u32 end = run.end - begin < r.per ? run.end : begin + r.per;
    if (at >= r.k) return;
    const u32 from = at + V <= r.k ? at : r.k - V, first = at - from;
    float dgain[V] = {}, dshift[V] = {};
    for (u32 row0 = begin; row0 < end; row0 += kRows) {
        Vec<T> x[kRows], dy[kRows];
        f32x4 m[kRows];
#pragma unroll
        for (u32 i = 0; i < kRows; ++i) {
            const u64 row = row0 + i < end ? row0 + i : row0;
            x[i] = load_any<Vec<T>>(static_cast<const T *>(r.x) + row * r.ldx + from);
            dy[i] = load_any<Vec<T>>(static_cast<const T *>(r.dy) + row * r.lddy + from);
            m[i] = r.stats[row];
        }
#pragma unroll
        for (u32 i = 0; i < kRows; ++i) {
            if (row0 + i >= end) break;
#pragma unroll
            for (u32 e = 0; e < V; ++e) {
                const float g = to_f32(dy[i][e]);
                dgain[e] += g * ((__builtin_fmaf(to_f32(x[i][e]), m[i][0], -m[i][1]) - m[i][2]) * m[i][3]);
                dshift[e] += g;
            }
        }
    }
    RowSlices all;
    all.init(r.offsets, r.blocks, r.rows, r.per);
    const bool alone = run.end - run.begin <= r.per;
    float *set = r.part + (u64)(run.block + all.slice_of(run.begin) + run.local) * 2 * r.k;
    float *to_gain = alone ? r.dgain ? r.dgain + (u64)run.block * r.k : nullptr : set;
    float *to_shift = alone ? r.dshift ? r.dshift + (u64)run.block * r.k : nullptr : set + r.k;
#pragma unroll
    for (u32 e = 0; e < V; ++e) {
        if (e < first) continue;
        if (to_gain) to_gain[from + e] = dgain[e];
        if (to_shift) to_shift[from + e] = dshift[e];
    }
}
u32 long_pieces(u32 k, u32 dtype) { return (k + 256 * (dtype == LMK_GS_F32 ? 4 : 8) - 1) / (256 * (dtype == LMK_GS_F32 ? 4 : 8)); }

// ---- launches

// How the threads share a row of k values: the fewest that hold it, with at most 16 values a thread (each stands in five registers in the
// gradients), and 8 where a workgroup of 1024 leaves a thread 128 registers.
struct NormShape {
    u32 g, c;               // threads of a row, vectors of a thread; g = 0: longer than registers
};
NormShape norm_shape(u32 k, u32 dtype, bool backward)
{
    const bool f32 = dtype == LMK_GS_F32;
    const u32 v = f32 ? 4 : 8, n = (k + v - 1) / v;
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {16, 2};
    if (n <= 64) return {64, 1};
    if (n <= 128) return {64, 2};
    if (n <= 256) return f32 ? NormShape{64, 4} : NormShape{256, 1};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return f32 ? NormShape{256, 4} : NormShape{1024, 1};
    if (k <= 8192 || (!backward && k <= 16384)) return {1024, (n + 1023) / 1024 > 2 ? 4u : 2u};
    return {0, 0};
}

// Rows of a run: whole turns of the rows that run beside each other.  Forward, eight workgroups a compute unit hide each other's loads (20 000 x 2000
// in bfloat16, eight / four / two: 29 / 32 / 42 us); those of 1024 threads all run at once, two a compute unit or, of more than eight values a thread,
// one (2889 x 4201 in bfloat16, eight / two / one: 25 / 21 / 24; 3000 x 12 000 48 / 37 / 33).  Of the gradients' runs as many as are held at once,
// and where that makes them short, fewer: a run's sums are written and read again (2 k floats), and joined one after the other.  A turn of a
// wavefront's rows is two chains of exchanges, of a workgroup's rows two meetings.
u32 norm_per(u32 rows, u32 blocks, u32 k, u32 dtype, bool backward)
{
    const NormShape s = norm_shape(k, dtype, backward);
    const u32 at_once = s.g == 0 ? 1 : threads_of(s.g) / s.g;
    const auto turns_of = [&](u32 workgroups) {
        const u64 t = ((u64)rows + (u64)workgroups * at_once - 1) / ((u64)workgroups * at_once);
        return (u32)(t < 1 ? 1 : t);
    };
    if (!backward) return turns_of(s.g < 1024 ? 2048 : s.c * (dtype == LMK_GS_F32 ? 4 : 8) <= 8 ? 512 : 256) * at_once;
    // of rows longer than registers: the sums' workgroups fill the device four times, with 16 rows or more (all gradients of 4096 rows of 16 000 in
    // bfloat16 466 us)
    if (s.g == 0) {
        const u32 runs = 1024 / long_pieces(k, dtype), per = turns_of(runs < 1 ? 1 : runs);
        return per < 16 ? 16 : per;
    }
    const u32 values = s.c * (dtype == LMK_GS_F32 ? 4 : 8), held = 256 * (s.g == 1024 ? 1 : values <= 8 ? 5 : 3);
    const double turn_us = s.g <= 64 ? 0.5 : s.g == 256 ? 0.8 : 1.2, set_us = 16.0 * k / 4e6;
    u32 best = 1;
    double least = -1;
    for (u32 turns = turns_of(held - (blocks < held / 2 ? blocks : held / 2)), i = 0; i < 8; ++i, turns *= 2) {
        const double runs = (double)rows / ((double)turns * at_once) + 1;
        const double us = turns * turn_us + runs * set_us + runs / blocks / 256 * 0.6;
        if (least < 0 || us < least) {
            least = us;
            best = turns;
        }
    }
    return best * at_once;
}

template <class T, bool BACKWARD, u32 G, u32 C>
hipError_t norm_go(const NormArgs &r, bool sums, hipStream_t stream)
{
    const dim3 grid((u32)max_runs(r.rows, r.blocks, r.per)), block(threads_of(G));
    if constexpr (BACKWARD) {
        if (sums) hipLaunchKernelGGL((norm_backward_kernel<T, G, C, true>), grid, block, 0, stream, r);
        else hipLaunchKernelGGL((norm_backward_kernel<T, G, C, false>), grid, block, 0, stream, r);
    } else {
        hipLaunchKernelGGL((norm_kernel<T, G, C>), grid, block, 0, stream, r);
    }
    return hipGetLastError();
}

template <class T, bool BACKWARD>
hipError_t norm_as(const NormArgs &r, hipStream_t stream)
{
    const bool sums = r.dgain || r.dshift;
    const NormShape s = norm_shape(r.k, std::is_same<T, float>::value ? LMK_GS_F32 : LMK_GS_BF16, BACKWARD);
    constexpr bool kF32 = std::is_same<T, float>::value;
    switch (s.g * 8 + s.c) {
    case 8 * 8 + 1: return norm_go<T, BACKWARD, 8, 1>(r, sums, stream);
    case 16 * 8 + 1: return norm_go<T, BACKWARD, 16, 1>(r, sums, stream);
    case 16 * 8 + 2: return norm_go<T, BACKWARD, 16, 2>(r, sums, stream);
    case 64 * 8 + 1: return norm_go<T, BACKWARD, 64, 1>(r, sums, stream);
    case 64 * 8 + 2: return norm_go<T, BACKWARD, 64, 2>(r, sums, stream);
    case 64 * 8 + 4: if constexpr (kF32) return norm_go<T, BACKWARD, 64, 4>(r, sums, stream); break;
    case 256 * 8 + 1: if constexpr (!kF32) return norm_go<T, BACKWARD, 256, 1>(r, sums, stream); break;
    case 256 * 8 + 2: return norm_go<T, BACKWARD, 256, 2>(r, sums, stream);
    case 256 * 8 + 4: if constexpr (kF32) return norm_go<T, BACKWARD, 256, 4>(r, sums, stream); break;
    case 1024 * 8 + 1: if constexpr (!kF32) return norm_go<T, BACKWARD, 1024, 1>(r, sums, stream); break;
    case 1024 * 8 + 2: if constexpr (kF32 || !BACKWARD) return norm_go<T, BACKWARD, 1024, 2>(r, sums, stream); break;
    case 1024 * 8 + 4: if constexpr (kF32 && !BACKWARD) return norm_go<T, BACKWARD, 1024, 4>(r, sums, stream); break;
    }
    const auto rows_go = [&](const NormArgs &a) {
        hipLaunchKernelGGL((long_norm_kernel<T, BACKWARD>), dim3(a.rows), dim3(kLong), 0, stream, a);
        return hipGetLastError();
    };
    if (!BACKWARD || !sums) return rows_go(r);
    // dx may take the place of what the sums read: statistics, sums, then dx
    NormArgs stats = r;
    stats.out = nullptr;
    hipError_t e = rows_go(stats);
    if (e != hipSuccess) return e;
    const u32 pieces = long_pieces(r.k, kF32 ? LMK_GS_F32 : LMK_GS_BF16);
    hipLaunchKernelGGL(long_norm_sums_kernel<T>, dim3(pieces * (u32)max_runs(r.rows, r.blocks, r.per)), dim3(256), 0, stream, r);
    e = hipGetLastError();
    return e == hipSuccess && r.out ? rows_go(r) : e;
}

NormArgs norm_args(const lmk_gs_norm &n, const void *x, u64 ldx, void *out, u64 ldo, bool backward)
{
    NormArgs r = {};
    r.x = x; r.ldx = ldx;
    r.gain = n.gain; r.shift = n.shift;
    r.offsets = n.offsets; r.blocks = n.blocks; r.rows = n.rows; r.k = n.k; r.eps = n.eps;
    r.out = out; r.ldo = ldo;
    r.per = norm_per(n.rows, n.blocks, n.k, n.dtype, backward);
    return r;
}

// sets of partial sums
u64 norm_sets(const lmk_gs_norm &n) { return (u64)n.rows / norm_per(n.rows, n.blocks, n.k, n.dtype, true) + n.blocks + 1; }
size_t norm_sets_bytes(const lmk_gs_norm &n) { return (size_t)(norm_sets(n) * 2 * n.k * 4 + 255) / 256 * 256; }

}  // namespace

bool grouped_norm_fits(const lmk_gs_norm &n, bool backward, bool sums)
{
    const NormShape s = norm_shape(n.k, n.dtype, backward);
    const u64 runs = max_runs(n.rows, n.blocks, norm_per(n.rows, n.blocks, n.k, n.dtype, backward));
    if (s.g == 0 ? (u64)n.rows * kLong >= kMostThreads : runs * threads_of(s.g) >= kMostThreads) return false;
    if (s.g == 0 && sums && runs * long_pieces(n.k, n.dtype) * 256 >= kMostThreads) return false;
    return !sums || join_threads(n.k, 1, n.blocks, (u32)(norm_sets(n) - n.blocks)) < kMostThreads;
}

size_t grouped_norm_backward_bytes(const lmk_gs_norm &n)
{
    return norm_sets_bytes(n) + (norm_shape(n.k, n.dtype, true).g == 0 ? (size_t)n.rows * sizeof(f32x4) : 0);
}

hipError_t launch_grouped_norm(const lmk_gs_norm &n, const void *x, u64 ldx, void *y, u64 ldy, hipStream_t stream)
{
    const NormArgs r = norm_args(n, x, ldx, y, ldy, false);
    return n.dtype == LMK_GS_F32 ? norm_as<float, false>(r, stream) : norm_as<__bf16, false>(r, stream);
}

hipError_t launch_grouped_norm_backward(const lmk_gs_norm &n, const void *dy, u64 lddy, const void *x, u64 ldx,
                                        const lmk_gs_norm_grads &out, char *workspace, hipStream_t stream)
{
    NormArgs r = norm_args(n, x, ldx, out.dx, out.lddx, true);
    r.dy = dy; r.lddy = lddy;
    r.dgain = out.dgain; r.dshift = out.dshift;
    const bool sums = out.dgain || out.dshift;
    r.part = reinterpret_cast<float *>(workspace);
    r.stats = sums ? reinterpret_cast<f32x4 *>(workspace + norm_sets_bytes(n)) : nullptr;
    if (n.rows > 0) {
        const hipError_t e = n.dtype == LMK_GS_F32 ? norm_as<float, true>(r, stream) : norm_as<__bf16, true>(r, stream);
        if (e != hipSuccess) return e;
    }
    return sums ? launch_join(n.offsets, n.blocks, n.rows, r.per, r.part, n.k, 1, out.dgain, out.dshift, (u32)(norm_sets(n) - n.blocks), stream)
                : hipSuccess;
}

}  // namespace lmk
