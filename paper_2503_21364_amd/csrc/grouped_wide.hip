// Grouped layers in bfloat16: the same products as in grouped_linear.hip on the bfloat16 matrix instructions
// (v_mfma_f32_16x16x32_bf16: exact products, sums in 32 bits; only results are rounded, once).
//
// Bound by those instructions and by LDS, which feeds them: 8192 x 8192 x 8192 at 1000 (forward), 1260 (dx), 1210
// (dw) and 1030 - 1080 TFLOP/s (dw from the 8-bit form); the largest library product reaches 1268.  65 536 rows in 32 ragged blocks
// of 1024 x 1024 (137 GFLOP a product), the same inputs again and again: forward 167 us, dx 163, dw and db 210 with 37 of joining.
// There 1076 tiles take five rounds of 256 workgroups where 4.2 would do, and a round's first loads and last stores have no
// products beside them: the accumulators and two steps' fragments of a lane leave no registers for the next tile's.
// The gate of dx adds 45 us (208 from codes, 205 from values): a lane's codes and scales are asked for sixteen times a tile, each
// time behind the stores in front.  The 8-bit form of x adds 36 (203; by itself it takes 64): its arithmetic stands between a
// meeting of the wavefronts and the products, for all of them at once.
//
// Tiles of 256 x 256, two wavefronts a SIMD: LDS gives a step's fragments in less time than their products take, which it
// does not for 128 x 128 (65 536 x 1024 x 1024 in 8 blocks: 183 us, large tiles 156) or 256 x 128 (slower than both).
#include "grouped.h"
#include "grouped_kernels.h"

namespace lmk {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(4))) u32 u32x4;
typedef __attribute__((ext_vector_type(2))) u32 u32x2;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

constexpr u32 kStep = 32;                   // sum indices of a matrix instruction
constexpr u32 kPair = 2 * kStep;            // of a filled part of LDS: 128 bytes of a row, a whole line
constexpr u32 kNowhere = 0x7ffffff0u;       // a byte offset behind every buffer below: reads give zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, u32 bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}

// ---- an operand of `W` rows (columns) by kPair sum indices in LDS, 128 W bytes, filled by loads that go to LDS
// directly (16 bytes a lane, 1 KB a wavefront, consecutive in LDS), one pair of steps after the other; what is out of range arrives as zeros.

// sum index contiguous in memory.  LDS: rows of eight 16-byte chunks, chunk c of row r in place c ^ (r / 2 % 8).  A 16-byte
// read is served 16 lanes at a time, lanes 0-3, 12-15 and 20-27, then the others of 32: they hold eight rows at one
// chunk and the other eight at the next, and are in 16 different places modulo 256 bytes.
template <u32 W, u32 WAVES> struct Along16 {
    static constexpr bool kDirect = true;
    static constexpr u32 kLoads = W / 8 / WAVES;
    const char *p;          // first row, first sum index
    u32 bytes;              // to the end of the last row
    u32 sums, s0;
    u32 from[kLoads];       // byte offset of this lane's chunk, sum index 0
    u32 s_lane;             // its first sum index in a pair of steps
    u32 read;               // LDS byte offset of this lane's part of the first 16 rows

    __device__ __forceinline__ void init(const __bf16 *base, u64 ld, u32 rows, u32 sums_, u32 wave, u32 lane)
    {
        p = reinterpret_cast<const char *>(base);
        sums = sums_;
        s0 = 0;
        bytes = ((rows - 1) * (u32)ld + sums) * 2;
        const u32 chunk = (lane & 7) ^ (lane >> 4) ^ (wave & 1) * 4;
        s_lane = chunk * 8;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) from[i] = ((wave + WAVES * i) * 8 + lane / 8) * (u32)ld * 2 + chunk * 16;
        read = (lane & 15) * 128 + (((lane >> 4) ^ (lane >> 1 & 7)) * 16);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32 wave)
    {
        const __amdgpu_buffer_rsrc_t b = buffer_of(p, bytes);
        const bool there = s0 + s_lane < sums;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, lds + (wave + WAVES * i) * 1024, 16, (int)(there ? from[i] + s0 * 2 : kNowhere), 0, 0, 0);
        s0 += kPair;
    }
    // half h of the pair; rows 16 f .. 16 f + 15 from the wavefront's first row r0 on
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const
    {
        return *reinterpret_cast<const lds_bf16x8 *>(lds + (read ^ h * 64) + (r0 + 16 * f) * 128);
    }
};

// rows (columns) contiguous in memory.  LDS: kPair rows of W values; 16 values (32 bytes) are a pair of chunks, pair p of sum
// index s in place p ^ g(s), g = s % 4 + 4 (s / 8 % 2): the eight sum indices whose rows half a wavefront reads in a
// transposed load have eight different g, so the pairs are in different places modulo 256 bytes.
__device__ __forceinline__ u32 turn(u32 s) { return (s & 3) | ((s >> 3 & 1) << 2); }

template <u32 W> __device__ __forceinline__ u32 across_read(u32 lane)
{
    const u32 s = 8 * (lane >> 4) + (lane >> 2 & 3);
    return s * (W * 2) + (turn(s) << 5) + (lane & 3) * 8;
}
// Four sum indices of one column.  `restrict` tells the compiler that the loads on their way into LDS go elsewhere (the barriers
// see to that); without it, it waits for all of them in front of every such read.
__device__ __forceinline__ s16x4 read_turned(const lds_char *__restrict__ a) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)a); }

template <u32 W> __device__ __forceinline__ bf16x8 across_fragment(const lds_char *lds, u32 read, u32 r0, u32 f)
{
    // a lane's 16-lane group turns four rows of 16 values: twice four sum indices of one column
    const lds_char *a = lds + (read ^ ((r0 / 16 + f) << 5));
    const s16x4 lo = read_turned(a), hi = read_turned(a + 4 * W * 2);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <u32 W, u32 WAVES> struct Across16 {
    static constexpr bool kDirect = true;
    static constexpr u32 kLoads = W / 8 / WAVES;
    u64 next;               // address of the next pair's first row (uniform)
    u32 left;               // its rows and all behind it
    u32 ld_bytes, width_bytes;
    u32 from[kLoads];
    u32 read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 ld, u32 width, u32 sums, u32 wave, u32 lane)
    {
        next = uniform64(reinterpret_cast<u64>(base));
        left = uniform(sums);
        ld_bytes = uniform((u32)ld * 2);
        width_bytes = uniform(width * 2);
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            const u32 at = (wave + WAVES * i) * 64 + lane, s = at / (W / 8), slot = at % (W / 8);
            const u32 chunk = ((slot >> 1) ^ turn(s)) * 2 + (slot & 1);
            from[i] = chunk * 8 < width ? s * ld_bytes + chunk * 16 : kNowhere;
        }
        read = across_read<W>(lane);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32 wave)
    {
        const u32 rows = left < kPair ? left : kPair;
        const __amdgpu_buffer_rsrc_t b = buffer_of(reinterpret_cast<const void *>(next), rows ? (rows - 1) * ld_bytes + width_bytes : 0u);
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b, lds + (wave + WAVES * i) * 1024, 16, (int)from[i], 0, 0, 0);
        next += (u64)kPair * ld_bytes;
        left -= rows;
    }
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const { return across_fragment<W>(lds + h * kStep * W * 2, read, r0, f); }
};

// ---- the same operands where rows start anywhere and end anywhere: through registers, one pair of steps ahead.

// eight bfloat16, moved down by d places (zeros come in)
__device__ __forceinline__ u32x4 move_down(u32x4 v, u32 d)
{
    u64 lo = (u64)v[1] << 32 | v[0], hi = (u64)v[3] << 32 | v[2];
    if (d >= 8) return u32x4{0, 0, 0, 0};
    if (d >= 4) {
        lo = hi >> (16 * (d - 4));
        hi = 0;
    } else if (d > 0) {
        lo = lo >> (16 * d) | hi << (64 - 16 * d);
        hi >>= 16 * d;
    }
    return u32x4{(u32)lo, (u32)(lo >> 32), (u32)hi, (u32)(hi >> 32)};
}

// sums >= 8: the last, partial eight of a row are read as its last whole ones
template <u32 W, u32 WAVES> struct AlongAny {
    static constexpr bool kDirect = false;
    static constexpr u32 kLoads = W / 8 / WAVES;
    const __bf16 *p;
    u32 sums, s0, chunk;
    u32 from[kLoads];       // offset of this thread's rows
    u32x4 v[kLoads];
    u32 to, read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 ld, u32 rows, u32 sums_, u32 wave, u32 lane)
    {
        p = base;
        sums = sums_;
        s0 = 0;
        const u32 thread = wave * kWave + lane, row = thread / 8;
        chunk = thread & 7;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) from[i] = (row + WAVES * 8 * i < rows ? row + WAVES * 8 * i : 0u) * (u32)ld;
        // WAVES * 8 rows further on, the chunks are turned alike
        to = row * 128 + ((chunk ^ (row >> 1 & 7)) * 16);
        read = (lane & 15) * 128 + (((lane >> 4) ^ (lane >> 1 & 7)) * 16);
        request();
    }
    __device__ __forceinline__ void request()
    {
        const u32 s = s0 + chunk * 8, at = s + 8 <= sums ? s : sums - 8;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) v[i] = load_any<u32x4>(p + from[i] + at);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32)
    {
        const u32 s = s0 + chunk * 8, d = s + 8 <= sums ? 0u : s - (sums - 8);
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            u32x4 o = v[i];
            if (s0 + kPair > sums) o = move_down(o, d);
            *reinterpret_cast<lds_u32x4 *>(lds + to + i * WAVES * 1024) = o;
        }
        s0 += kPair;
        request();
    }
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const
    {
        return *reinterpret_cast<const lds_bf16x8 *>(lds + (read ^ h * 64) + (r0 + 16 * f) * 128);
    }
};

// rows of eight columns and more
template <u32 W, u32 WAVES> struct AcrossAny {
    static constexpr bool kDirect = false;
    static constexpr u32 kLoads = W / 8 / WAVES, kRows = WAVES * kWave * 8 / W;      // rows of a turn of loads
    static_assert(kRows % 16 == 0, "rows of another turn are turned alike");
    const __bf16 *p;        // this thread's columns of the next pair's first row
    u64 ld;
    u32 left, row, d;
    u32x4 v[kLoads];
    u32 to, read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 ld_, u32 width, u32 sums, u32 wave, u32 lane)
    {
        const u32 thread = wave * kWave + lane, chunk = thread % (W / 8), col = chunk * 8;
        row = thread / (W / 8);
        ld = ld_;
        left = sums;
        // columns behind the last one are anything: their results are not kept
        const int at = col + 8 <= width ? (int)col : (int)width - 8;
        d = (u32)((int)col - at);
        p = base + at;
        to = row * (W * 2) + ((((chunk >> 1) ^ turn(row)) * 2 + (chunk & 1)) * 16);
        read = across_read<W>(lane);
        request();
    }
    __device__ __forceinline__ void request()
    {
        if (left == 0) return;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) v[i] = load_any<u32x4>(p + (row + kRows * i < left ? row + kRows * i : 0u) * ld);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32)
    {
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            u32x4 o = v[i];
            if (d > 0) o = move_down(o, d);
            if (row + kRows * i >= left) o = u32x4{0, 0, 0, 0};
            *reinterpret_cast<lds_u32x4 *>(lds + to + i * kRows * W * 2) = o;
        }
        p += (u64)kPair * ld;
        left = left > kPair ? left - kPair : 0u;
        request();
    }
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const { return across_fragment<W>(lds + h * kStep * W * 2, read, r0, f); }
};

// Tile of TP x TQ results: P runs along the output's contiguous axis (a lane holds four consecutive ones of it), Q across it.
template <u32 TP, u32 TQ, u32 WP, u32 WQ> struct Shape {
    static constexpr u32 kWaves = WP * WQ, kThreads = kWaves * kWave;
    static constexpr u32 kP = TP / WP / 16, kQ = TQ / WQ / 16;           // 16 x 16 results of a wavefront
    static constexpr u32 kPartP = TP * kPair * 2, kPartQ = TQ * kPair * 2, kLds = 2 * (kPartP + kPartQ);
    static constexpr u32 kResident = 512 / kThreads;                     // workgroups of a compute unit
};

// The wavefronts meet, each with no more loads and LDS accesses on their way than WAIT says.  Neither builtin promises an order to the
// memory accesses around it: the two empty statements keep stores to LDS in front of the meeting and reads behind it.
template <u32 WAIT> __device__ __forceinline__ void wavefronts_meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(WAIT);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// acc[i][j] += P Q over `steps`.  LDS holds two pairs of steps.  A step's fragments are read from LDS while the step in front of
// it is multiplied; once the second step's are with all wavefronts, the pair's part is filled again, which has the
// time of two steps to arrive.  One meeting of the wavefronts a pair.
// `also` sees the fragments of Q, `look` a pair of steps of Q in LDS.
template <class S, class P, class Q, class Also, class Look>
__device__ __forceinline__ void wide_product(P &p, Q &q, u32 steps, lds_char *lds, u32 wave, u32 p0, u32 q0,
                                             f32x4 (&acc)[S::kP][S::kQ], Also &&also, Look &&look)
{
    lds_char *lp = lds, *lq = lds + 2 * S::kPartP;
    constexpr bool kDirect = P::kDirect && Q::kDirect;
    if constexpr (kDirect) static_assert(P::kLoads + Q::kLoads == 8, "the wait below counts eight loads a pair");
    bf16x8 fp[S::kP], fq[2][S::kQ];
    auto fill = [&](u32 part) {
        p.fill(lp + part * S::kPartP, wave);
        q.fill(lq + part * S::kPartQ, wave);
    };
    // multiplies step h and reads the fragments of half `hn` of part `pn`: those of P take the place of what has been used
    auto step = [&](u32 h, u32 pn, u32 hn) {
#pragma unroll
        for (u32 j = 0; j < S::kQ; ++j) fq[hn][j] = q.fragment(lq + pn * S::kPartQ, hn, q0, j);
#pragma unroll
        for (u32 i = 0; i < S::kP; ++i) {
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i], fq[h][j], acc[i][j], 0, 0, 0);
            fp[i] = p.fragment(lp + pn * S::kPartP, hn, p0, i);
        }
        also(fq[h]);
        asm volatile("" ::: "memory");              // the reads stay in this step
    };
    fill(0);
    fill(1);
    wavefronts_meet<kDirect ? 0xF70 | 8 : 0x070>();                 // the second pair's eight loads may be on their way
#pragma unroll
    for (u32 i = 0; i < S::kP; ++i) fp[i] = p.fragment(lp, 0, p0, i);
#pragma unroll
    for (u32 j = 0; j < S::kQ; ++j) fq[0][j] = q.fragment(lq, 0, q0, j);
    for (u32 t0 = 0; t0 < steps; t0 += 4) {
#pragma unroll
        for (u32 part = 0; part < 2; ++part) {
            const u32 t = t0 + 2 * part;
            if (t >= steps) break;
            look(t / 2, lq + part * S::kPartQ);
            step(0, part, 1);
            if (t + 1 >= steps) break;
            // the next pair has arrived, and this pair's fragments have left LDS
            wavefronts_meet<0x070>();
            fill(part);
            step(1, 1 - part, 0);
        }
    }
    // nothing may be on its way into LDS when the workgroup ends
    __builtin_amdgcn_s_waitcnt(0x070);
}

__device__ __forceinline__ u32 pack_bf16(float a, float b)
{
    return (u32)__builtin_bit_cast(unsigned short, (__bf16)a) | ((u32)__builtin_bit_cast(unsigned short, (__bf16)b) << 16);
}

// 32 values of a row of x, a thread's, from the pair of steps that is in LDS (laid out as Along16 does) to their 8-bit form.  They
// are read twice: held, they would cost registers that the products need.
__device__ __forceinline__ void keep_pair(const RowsArgs &r, const lds_char *lds, u32 pair, u32 row0, u32 height, u32 thread)
{
    const u32 row = thread / 2, half = thread & 1, kp = (r.sums + 31) / 32 * 32, col = pair * kPair + half * 32;
    if (row >= height || col >= kp) return;
    const lds_char *p = lds + row * 128;
    const u32 turned = row >> 1 & 7;
    const auto chunk = [&](u32 c) { return *reinterpret_cast<const lds_u32x4 *>(p + (((4 * half + c) ^ turned) * 16)); };
    u32 top = 0;
#pragma unroll
    for (u32 c = 0; c < 4; ++c) {
        const u32x4 v = chunk(c);
#pragma unroll
        for (u32 e = 0; e < 4; ++e) {
            const u32 lo = v[e] & 0x7fffu, hi = v[e] >> 16 & 0x7fffu;
            top = top > lo ? top : lo;
            top = top > hi ? top : hi;
        }
    }
    const u32 scale = scale_of_max(top << 16);
    const float inv = inverse_step(scale);
    const u64 at = (u64)(row0 + row) * kp + col;
#pragma unroll
    for (u32 h = 0; h < 2; ++h) {
        u32x4 o;
#pragma unroll
        for (u32 c = 0; c < 2; ++c) {
            const u32x4 v = chunk(2 * h + c);
#pragma unroll
            for (u32 e = 0; e < 2; ++e)
                o[2 * c + e] = pack_codes(code_of(__uint_as_float(v[2 * e] << 16), inv), code_of(__uint_as_float(v[2 * e] & 0xffff0000u), inv),
                                          code_of(__uint_as_float(v[2 * e + 1] << 16), inv), code_of(__uint_as_float(v[2 * e + 1] & 0xffff0000u), inv));
        }
        *reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(r.keep_codes) + at + 16 * h) = o;
    }
    r.keep_scale[at / 32] = (uint8_t)scale;
}

// GATE: 0 none, 1 values, 2 codes, 3 none, and the 8-bit form of x is written: whole lines of it, two pairs of steps of a row, by the
// workgroups of its columns in turn
template <class S, u32 TP, u32 TQ, u32 WP, bool ACROSS, bool ANY, u32 GATE>
__global__ __launch_bounds__(S::kThreads, 2) void wide_rows_kernel(const RowsArgs r)
{
    extern __shared__ __align__(16) char wide_lds[];
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, S::kResident * kUnits);
    const u32 row_tile = tile / r.col_tiles, col_tile = tile - row_tile * r.col_tiles, col0 = col_tile * TP;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, TQ, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * TQ;
    const u32 height = run.end - row0 < TQ ? run.end - row0 : TQ;
    const u32 width = r.cols - col0 < TP ? r.cols - col0 : TP;
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 p0 = wave % WP * (S::kP * 16), q0 = wave / WP * (S::kQ * 16);
    f32x4 acc[S::kP][S::kQ] = {};
    const bool inside = run.block != ~0u;
    const auto nothing = [](const bf16x8 (&)[S::kQ]) {};
    const auto keep = [&](u32 pair, const lds_char *lds) {
        if (GATE == 3 && pair / 2 % r.col_tiles == col_tile) keep_pair(r, lds, pair, row0, height, threadIdx.x);
    };
    if (GATE == 3 && !inside && col_tile == 0) {
        const u32 kp = (r.sums + 31) / 32 * 32;
        for (u32 i = threadIdx.x; i < height * (kp / 32); i += S::kThreads) {
            u32x4 *p = reinterpret_cast<u32x4 *>(reinterpret_cast<char *>(r.keep_codes) + (u64)row0 * kp) + (u64)i * 2;
            p[0] = p[1] = u32x4{0, 0, 0, 0};
            r.keep_scale[(u64)row0 * (kp / 32) + i] = 0;
        }
    }
    if (inside) {
        lds_char *lds = (lds_char *)wide_lds;
        const u32 steps = (r.sums + kStep - 1) / kStep;
        typename std::conditional<ANY, AlongAny<TQ, S::kWaves>, Along16<TQ, S::kWaves>>::type q;
        q.init(static_cast<const __bf16 *>(r.a) + (u64)row0 * r.lda, r.lda, height, r.sums, wave, lane);
        const __bf16 *w = static_cast<const __bf16 *>(r.w) + (u64)run.block * r.w_block;
        if constexpr (ACROSS) {
            typename std::conditional<ANY, AcrossAny<TP, S::kWaves>, Across16<TP, S::kWaves>>::type p;
            p.init(w + col0, r.ldw, width, r.sums, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, nothing, keep);
        } else {
            typename std::conditional<ANY, AlongAny<TP, S::kWaves>, Along16<TP, S::kWaves>>::type p;
            p.init(w + (u64)col0 * r.ldw, r.ldw, width, r.sums, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, nothing, keep);
        }
    }
    // Two neighbouring results exchange lanes, so that a lane has eight consecutive values of a row:
    // lane group 0: the first eight of result i, 1: of i + 1, 2 and 3: the second eight.
    const u32 group = lane >> 4;
    __bf16 *out = static_cast<__bf16 *>(r.out) + (u64)row0 * r.ldo + col0;
#pragma unroll
    for (u32 i = 0; i < S::kP; i += 2) {
        const u32 c_own = p0 + 16 * i + 4 * group;           // of result i, before the exchange
        f32x4 bias[2] = {};
        if (r.bias && inside) {
            const float *b = r.bias + (u64)run.block * r.cols + col0;
#pragma unroll
            for (u32 h = 0; h < 2; ++h)
#pragma unroll
                for (u32 v = 0; v < 4; ++v) {
                    const u32 c = c_own + 16 * h + v;
                    bias[h][v] = c < width ? b[c] : 0.0f;
                }
        }
        const u32 c = p0 + 16 * (i + (group & 1)) + 8 * (group >> 1);
#pragma unroll
        for (u32 j = 0; j < S::kQ; ++j) {
            f32x4 y[2] = {acc[i][j] + bias[0], acc[i + 1][j] + bias[1]};
            if (r.relu) {
#pragma unroll
                for (u32 v = 0; v < 4; ++v) {
                    y[0][v] = y[0][v] < 0.0f ? 0.0f : y[0][v];          // NaN stays
                    y[1][v] = y[1][v] < 0.0f ? 0.0f : y[1][v];
                }
            }
            const u32x2 a = __builtin_amdgcn_permlane16_swap(pack_bf16(y[0][0], y[0][1]), pack_bf16(y[1][0], y[1][1]), false, false);
            const u32x2 b = __builtin_amdgcn_permlane16_swap(pack_bf16(y[0][2], y[0][3]), pack_bf16(y[1][2], y[1][3]), false, false);
            u32x4 v = {a[0], b[0], a[1], b[1]};
            const u32 row = q0 + 16 * j + (lane & 15);
            if (row >= height || c >= width) continue;
            if (ANY && c + 8 > width) {
#pragma unroll
                for (u32 e = 0; e < 8; ++e) {
                    if (c + e >= width) continue;
                    const u64 at = (u64)(row0 + row) * r.ldgate + col0 + c + e;
                    bool pass = true;
                    if (GATE == 1 && inside) pass = !((float)static_cast<const __bf16 *>(r.gate)[at] <= 0.0f);
                    if (GATE == 2 && inside) pass = static_cast<const signed char *>(r.gate)[at] > 0 || r.gate_scale[at / 32] == 255;
                    out[(u64)row * r.ldo + c + e] = pass ? __builtin_bit_cast(__bf16, (unsigned short)(v[e / 2] >> (16 * (e % 2)))) : (__bf16)0.0f;
                }
                continue;
            }
            if (GATE == 1 && inside) {
                const bf16x8 x = load_any<bf16x8>(static_cast<const __bf16 *>(r.gate) + (u64)(row0 + row) * r.ldgate + col0 + c);
#pragma unroll
                for (u32 e = 0; e < 4; ++e) {
                    if ((float)x[2 * e] <= 0.0f) v[e] &= 0xffff0000u;
                    if ((float)x[2 * e + 1] <= 0.0f) v[e] &= 0x0000ffffu;
                }
            }
            if (GATE == 2 && inside) {
                const u64 at = (u64)(row0 + row) * r.ldgate + col0 + c;
                const u32x2 codes = *reinterpret_cast<const u32x2 *>(static_cast<const char *>(r.gate) + at);
                if (r.gate_scale[at / 32] != 255) {
#pragma unroll
                    for (u32 e = 0; e < 8; ++e)
                        if ((int)(signed char)(codes[e / 4] >> (8 * (e % 4))) <= 0) v[e / 2] &= e % 2 ? 0x0000ffffu : 0xffff0000u;
                }
            }
            store_any(out + (u64)row * r.ldo + c, v);
        }
    }
}

}  // namespace

namespace {

// ---- sums over rows

// x of the sums over rows from its 8-bit form.  A thread has the 32 codes of a row that share a step; they come to registers
// two pairs of steps ahead and are widened on their way into LDS (exactly: a code times a power of two), laid out as
// Across16 does.  fill() writes the next pair and requests the one behind it.
template <u32 W, u32 WAVES> struct Codes16 {
    static constexpr bool kDirect = false;
    static_assert(kPair * W / 32 == WAVES * kWave, "one group of 32 codes a thread");
    const char *codes;      // this thread's codes of the next pair of steps
    const uint8_t *scale;
    u32 kp, row, rows;
    bool there;
    u32 read, to[2];
    u32x4 v[2];
    u32 e;

    __device__ __forceinline__ void init(const char *codes_, const uint8_t *scale_, u32 kp_, u32 width, u32 sums, u32 wave, u32 lane)
    {
        const u32 thread = wave * kWave + lane, group = thread % (W / 32);
        row = thread / (W / 32);
        kp = kp_;
        rows = sums;
        there = group * 32 < width;
        codes = codes_ + (u64)row * kp + group * 32;
        scale = scale_ + (u64)row * (kp / 32) + group;
        read = across_read<W>(lane);
#pragma unroll
        for (u32 i = 0; i < 2; ++i) to[i] = row * (W * 2) + (((2 * group + i) ^ turn(row)) << 5);
        request();
    }
    __device__ __forceinline__ void request()
    {
        v[0] = v[1] = u32x4{0, 0, 0, 0};
        e = 0;
        if (there && row < rows) {
            v[0] = reinterpret_cast<const u32x4 *>(codes)[0];
            v[1] = reinterpret_cast<const u32x4 *>(codes)[1];
            e = *scale;
        }
        row += kPair;
        codes += (u64)kPair * kp;
        scale += (u64)kPair * (kp / 32);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32)
    {
        const float step = step_of(e);
#pragma unroll
        for (u32 i = 0; i < 4; ++i) {
            u32x4 o;
#pragma unroll
            for (u32 h = 0; h < 4; ++h) {
                const u32 q = v[i / 2][i % 2 * 2 + h / 2] >> (16 * (h % 2));
                o[h] = pack_bf16(value_of(q, 0, step), value_of(q, 1, step));
            }
            *reinterpret_cast<lds_u32x4 *>(lds + to[i / 2] + 16 * (i % 2)) = o;
        }
        request();
    }
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const { return across_fragment<W>(lds + h * kStep * W * 2, read, r0, f); }
};

// Tiles of dw over a slice of the rows: P = x (inputs), Q = dy (outputs).  db rides on the tiles of the first inputs: a
// matrix instruction with ones in the place of x, the wavefronts along P taking turns.
template <class S, u32 TP, u32 TQ, u32 WP, bool CODES, bool ANY>
__global__ __launch_bounds__(S::kThreads, 2) void wide_sums_kernel(const SumsArgs r)
{
    extern __shared__ __align__(16) char wide_lds[];
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, S::kResident * kUnits);
    const u32 pairs = r.n_tiles * r.k_tiles, slice = tile / pairs, pair = tile - slice * pairs;
    const u32 n0 = pair / r.k_tiles * TQ, k0 = pair % r.k_tiles * TP;
    const u32 height = r.n - n0 < TQ ? r.n - n0 : TQ, width = r.k - k0 < TP ? r.k - k0 : TP;
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 pw = wave % WP, p0 = pw * (S::kP * 16), q0 = wave / WP * (S::kQ * 16);
    const bool sums_db = r.db && k0 == 0;
    constexpr u32 kB = (S::kQ + WP - 1) / WP;
    lds_char *lds = (lds_char *)wide_lds;
    SliceRuns run;
    run.init(r.offsets, r.blocks, r.rows, r.per, slice);
    while (run.next()) {
        const u32 lane = afresh(threadIdx.x & (kWave - 1));
        f32x4 acc[S::kP][S::kQ] = {};
        f32x4 bias[kB] = {};
        __syncthreads();                    // the run in front of this one is out of LDS
        const u32 steps = (run.count + kStep - 1) / kStep;
        const __bf16 one = (__bf16)1.0f;
        const bf16x8 ones = {one, one, one, one, one, one, one, one};
        const auto add = [&](const bf16x8 (&fq)[S::kQ]) {
            if (!sums_db) return;
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j)
                if (j % WP == pw) bias[j / WP] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fq[j], bias[j / WP], 0, 0, 0);
        };
        typename std::conditional<ANY, AcrossAny<TQ, S::kWaves>, Across16<TQ, S::kWaves>>::type q;
        q.init(static_cast<const __bf16 *>(r.dy) + (u64)run.row * r.lddy + n0, r.lddy, height, run.count, wave, lane);
        if constexpr (CODES) {
            const u32 kp = (r.k + 31) / 32 * 32;
            Codes16<TP, S::kWaves> p;
            p.init(static_cast<const char *>(r.x) + (u64)run.row * kp + k0, r.scale + (u64)run.row * (kp / 32) + k0 / 32, kp, kp - k0,
                   run.count, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, add, [](u32, const lds_char *) {});
        } else {
            typename std::conditional<ANY, AcrossAny<TP, S::kWaves>, Across16<TP, S::kWaves>>::type p;
            p.init(static_cast<const __bf16 *>(r.x) + (u64)run.row * r.ldx + k0, r.ldx, width, run.count, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, add, [](u32, const lds_char *) {});
        }
        const u64 size = (u64)r.n * r.k;
        float *dw = run.whole ? r.dw + (u64)run.block * size : r.part + (u64)run.partial() * (size + r.n);
        float *db = run.whole ? r.db + (u64)run.block * r.n : r.part + (u64)run.partial() * (size + r.n) + size;
#pragma unroll
        for (u32 j = 0; j < S::kQ; ++j) {
            const u32 n = n0 + q0 + 16 * j + (lane & 15);
            if (n >= r.n) continue;
#pragma unroll
            for (u32 i = 0; i < S::kP; ++i) {
                const u32 k = k0 + p0 + 16 * i + 4 * (lane >> 4);
                if (k >= r.k) continue;
                if (r.in_major || (ANY && k + 4 > r.k)) {
#pragma unroll
                    for (u32 v = 0; v < 4; ++v)
                        if (!ANY || k + v < r.k) dw[r.in_major ? (u64)(k + v) * r.n + n : (u64)n * r.k + k + v] = acc[i][j][v];
                } else {
                    store_any(dw + (u64)n * r.k + k, acc[i][j]);
                }
            }
            if (sums_db && j % WP == pw && lane < 16) db[n] = bias[j / WP][0];
        }
    }
}

// ---- launches

template <u32 TP, u32 TQ, u32 WP, u32 WQ, bool ACROSS, bool ANY, u32 GATE>
hipError_t wide_go(RowsArgs r, hipStream_t stream)
{
    using S = Shape<TP, TQ, WP, WQ>;
    r.col_tiles = (r.cols + TP - 1) / TP;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, TQ) * r.col_tiles);
    auto kernel = wide_rows_kernel<S, TP, TQ, WP, ACROSS, ANY, GATE>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(r.tiles), dim3(S::kThreads), S::kLds, stream, r);
    return hipGetLastError();
}
bool sixteen(const void *p, u64 ld) { return ld % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0; }

bool rows_sixteen(const RowsArgs &r)
{
    return r.sums % 8 == 0 && r.cols % 8 == 0 && sixteen(r.a, r.lda) && sixteen(r.w, r.ldw) && r.w_block % 8 == 0;
}

// Which tiles, from the rounds that the device's compute units take (all blocks but one end half a tile early in the mean).  Of 256 x 256
// tiles a round is 256, and its costs come whole; of 128 x 128 it is 512, two workgroups a compute unit, with 0.7 of the time
// for half of the results, and the two even out what a last round leaves.  8 ragged blocks of 1024 x 1024, large / small tiles: 4096 rows
// 30 / 20 us, 16 384 56 / 48, 65 536 158 / 183; one of 512 x 512: 16 384 20 / 14, 32 768 23 / 31.
bool large_tiles(const RowsArgs &r)
{
    const auto share = [&](u32 side) { return __builtin_ceilf((float)r.rows / side + 0.5f * (r.blocks - 1)) * ((r.cols + side - 1) / side); };
    return __builtin_ceilf(share(256) / 256) < 0.7f * share(128) / 512;
}

template <bool ACROSS, u32 GATE>
hipError_t wide_shape(const RowsArgs &r, hipStream_t stream)
{
    if (!rows_sixteen(r)) return wide_go<128, 128, 2, 2, ACROSS, true, GATE>(r, stream);
    if (large_tiles(r)) return wide_go<256, 256, 2, 4, ACROSS, false, GATE>(r, stream);
    return wide_go<128, 128, 2, 2, ACROSS, false, GATE>(r, stream);
}

bool sums_sixteen(const SumsArgs &r)
{
    return r.n % 8 == 0 && sixteen(r.dy, r.lddy) && (r.scale || (r.k % 8 == 0 && sixteen(r.x, r.ldx))) && r.k % 4 == 0;
}

template <u32 TP, u32 TQ, u32 WP, u32 WQ, bool ANY>
hipError_t wide_sums_go(SumsArgs r, bool codes, hipStream_t stream)
{
    using S = Shape<TP, TQ, WP, WQ>;
    r.n_tiles = (r.n + TQ - 1) / TQ;
    r.k_tiles = (r.k + TP - 1) / TP;
    r.tiles = (u32)((u64)r.slices * r.n_tiles * r.k_tiles);
    auto kernel = codes ? wide_sums_kernel<S, TP, TQ, WP, true, ANY> : wide_sums_kernel<S, TP, TQ, WP, false, ANY>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(r.tiles), dim3(S::kThreads), S::kLds, stream, r);
    return hipGetLastError();
}

}  // namespace

// Offsets inside a tile are 32 bits wide.  Narrower than eight: the general kernel.
bool wide_rows_fit(const RowsArgs &r)
{
    constexpr u64 most = 1u << 21;
    return r.sums >= 8 && r.cols >= 8 && r.lda <= most && r.ldw <= most;
}

u64 wide_rows_threads(const RowsArgs &r)
{
    const u32 side = rows_sixteen(r) && large_tiles(r) ? 256 : 128;
    return max_runs(r.rows, r.blocks, side) * ((r.cols + side - 1) / side) * (side * 2);
}

hipError_t launch_wide_rows(const RowsArgs &r, bool across, hipStream_t stream)
{
    const u32 gate = r.keep_codes ? 3 : !r.gate ? 0 : r.gate_scale ? 2 : 1;
    if (gate == 3) return across ? wide_shape<true, 3>(r, stream) : wide_shape<false, 3>(r, stream);
    if (across) return gate == 0 ? wide_shape<true, 0>(r, stream) : gate == 1 ? wide_shape<true, 1>(r, stream) : wide_shape<true, 2>(r, stream);
    return gate == 0 ? wide_shape<false, 0>(r, stream) : gate == 1 ? wide_shape<false, 1>(r, stream) : wide_shape<false, 2>(r, stream);
}

bool wide_sums_fit(const SumsArgs &r)
{
    constexpr u64 most = 1u << 21;
    return r.n >= 8 && r.k >= 8 && r.lddy <= most && (r.scale || r.ldx <= most);
}

u64 wide_sums_threads(const SumsArgs &r)
{
    const u32 side = sums_sixteen(r) ? r.side : 128;
    return (u64)r.slices * ((r.n + side - 1) / side) * ((r.k + side - 1) / side) * (side * 2);
}

hipError_t launch_wide_sums(const SumsArgs &r, hipStream_t stream)
{
    if (!sums_sixteen(r)) return wide_sums_go<128, 128, 2, 2, true>(r, r.scale != nullptr, stream);
    if (r.side == 256) return wide_sums_go<256, 256, 2, 4, false>(r, r.scale != nullptr, stream);
    return wide_sums_go<128, 128, 2, 2, false>(r, r.scale != nullptr, stream);
}

}  // namespace lmk
