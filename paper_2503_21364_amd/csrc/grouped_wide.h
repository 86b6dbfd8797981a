// The product of a tile on the bfloat16 matrix instructions, and how its operands come into LDS.
#ifndef LMK_GS_GROUPED_WIDE_H
#define LMK_GS_GROUPED_WIDE_H
#include "grouped_kernels.h"

namespace lmk {

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
    // what the compiler does not see to be the same in all lanes costs a loop around every load
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(uniform64(reinterpret_cast<u64>(p))), 0, (int)uniform(bytes), 0x00020000);
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
// `also` sees the fragments of Q, `look` a pair of steps of Q in LDS.  STARTED: the first two pairs have been asked for, and the first is there.
template <class S, bool STARTED = false, class P, class Q, class Also, class Look>
__device__ __forceinline__ void wide_product(P &p, Q &q, u32 steps, lds_char *lds, u32 wave, u32 p0, u32 q0,
                                             f32x4 (&acc)[S::kP][S::kQ], Also &&also, Look &&look)
{
    lds_char *lp = lds, *lq = lds + 2 * S::kPartP;
    constexpr bool kDirect = P::kDirect && Q::kDirect;
    // the second pair's loads may be on their way
    constexpr u32 kFirst = [] {
        if constexpr (kDirect) {
            static_assert(P::kLoads + Q::kLoads < 16, "four bits of a count");
            return 0xF70u | (P::kLoads + Q::kLoads);
        } else {
            return 0x070u;
        }
    }();
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
    if constexpr (!STARTED) {
        fill(0);
        fill(1);
        wavefronts_meet<kFirst>();
    }
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

// Around the stores of a whole tile, of which the next tile's first wait counts N behind its loads: a remark in the compiler's output, where a test
// counts those that every lane reaches.  Fewer would end that wait before the loads are there.
template <u32 N> __device__ __forceinline__ void stores_begin() { asm volatile("; %0 stores begin" : : "n"(N) : "memory"); }
__device__ __forceinline__ void stores_end() { asm volatile("; stores end" : : : "memory"); }

// one conversion instruction
__device__ __forceinline__ u32 pack_bf16(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(u32, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Results of a launch that are more than the dies' caches hold together are stored past them: the operands stay there (y of 65 536 x 2048 from
// operands in 4 bits: 215 us, so 198).  Rows have to begin with whole lines: parts of one are not put together there (65 536 rows of 512 -> 1000 in
// 4 bits: 61 us, through the caches 45).
inline bool past_caches(const void *p, u64 row_bytes, u64 bytes)
{
    return bytes > 32u << 20 && row_bytes % 128 == 0 && reinterpret_cast<uintptr_t>(p) % 128 == 0;
}
// 16 bytes at any address
template <bool PAST, class T, class V> __device__ __forceinline__ void store_vector(T *p, V v)
{
    if constexpr (PAST) {
        typedef V any __attribute__((aligned(2)));
        __builtin_nontemporal_store(v, reinterpret_cast<any *>(p));
    } else {
        store_any(p, v);
    }
}

}  // namespace lmk
#endif
