// Gated layers in bfloat16 on the bfloat16 matrix instructions: the tiles of grouped_wide.hip, of whose rows of weights 16 are of the
// gate and the next 16 of the other projection, in turns.  A lane then has both projections of the same four outputs in neighbouring
// accumulators, and the activation, the product and their gradients need no exchange.
//
// Bound by the bfloat16 instructions and by LDS: y of 8192 rows of 8192 -> 4096 at 1446 TFLOP/s, of 16 384 rows of 2048 -> 4096 in 4 even blocks at 1370 (SiLU; GELU 1260);
// 65 536 rows of 1024 -> 2048 in 32 even blocks 491 us (1120), in ragged ones 510 to 546: a block's weights are read by eight or nine tiles of rows only, and a tile has 32 steps
// between its first loads and its last stores.  The gradients of both projections of the second take 545 us: the activation's arithmetic and two
// results for each of y's, with nothing of the products beside them.
#include "grouped_gated.h"
#include "grouped_wide.h"

namespace lmk {

namespace {

// Row (column) p of a tile of weights: output o of projection `second`
__device__ __forceinline__ u32 output_of(u32 p) { return p / 32 * 16 + p % 16; }
__device__ __forceinline__ bool second_of(u32 p) { return (p / 16 & 1) != 0; }

// As Along16, AlongAny, Across16 and AcrossAny, for the weights of both projections; `width`: outputs of the tile that there are.
template <u32 W, u32 WAVES> struct BothAlong16 {
    static constexpr bool kDirect = true;
    static constexpr u32 kLoads = W / 8 / WAVES;
    const char *p[2];
    u32 bytes, sums, s0;
    u32 from[kLoads];
    u32 s_lane, read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 second, u64 ld, u32 width, u32 sums_, u32 wave, u32 lane)
    {
        p[0] = reinterpret_cast<const char *>(base);
        p[1] = reinterpret_cast<const char *>(base + second);
        sums = sums_;
        s0 = 0;
        bytes = ((width - 1) * (u32)ld + sums) * 2;
        const u32 chunk = (lane & 7) ^ (lane >> 4) ^ (wave & 1) * 4;
        s_lane = chunk * 8;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) from[i] = output_of((wave + WAVES * i) * 8 + lane / 8) * (u32)ld * 2 + chunk * 16;
        read = (lane & 15) * 128 + (((lane >> 4) ^ (lane >> 1 & 7)) * 16);
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32 wave)
    {
        const __amdgpu_buffer_rsrc_t b[2] = {buffer_of(p[0], bytes), buffer_of(p[1], bytes)};
        const bool there = s0 + s_lane < sums;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            // eight rows a load, of one projection
            const u32 at = (wave + WAVES * i) * 8;
            if (second_of(at)) __builtin_amdgcn_raw_ptr_buffer_load_lds(b[1], lds + at * 128, 16, (int)(there ? from[i] + s0 * 2 : kNowhere), 0, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(b[0], lds + at * 128, 16, (int)(there ? from[i] + s0 * 2 : kNowhere), 0, 0, 0);
        }
        s0 += kPair;
    }
    __device__ __forceinline__ bf16x8 fragment(const lds_char *lds, u32 h, u32 r0, u32 f) const
    {
        return *reinterpret_cast<const lds_bf16x8 *>(lds + (read ^ h * 64) + (r0 + 16 * f) * 128);
    }
};

template <u32 W, u32 WAVES> struct BothAcross16 {
    static constexpr bool kDirect = true;
    static constexpr u32 kLoads = W / 8 / WAVES;
    u64 next;
    u32 left;
    u32 ld_bytes, width_bytes;
    u32 from[kLoads];
    u32 read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 second, u64 ld, u32 width, u32 sums, u32 wave, u32 lane)
    {
        next = uniform64(reinterpret_cast<u64>(base));
        left = uniform(sums);
        ld_bytes = uniform((u32)ld * 2);
        width_bytes = uniform(((u32)second + width) * 2);          // to the end of the second projection's columns
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            const u32 at = (wave + WAVES * i) * 64 + lane, s = at / (W / 8), slot = at % (W / 8);
            const u32 col = (((slot >> 1) ^ turn(s)) * 2 + (slot & 1)) * 8, o = output_of(col);
            from[i] = o < width ? s * ld_bytes + (o + (second_of(col) ? (u32)second : 0u)) * 2 : kNowhere;
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

template <u32 W, u32 WAVES> struct BothAlongAny {
    static constexpr bool kDirect = false;
    static constexpr u32 kLoads = W / 8 / WAVES;
    const __bf16 *p[kLoads];
    u32 sums, s0, chunk;
    u32x4 v[kLoads];
    u32 to, read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 second, u64 ld, u32 width, u32 sums_, u32 wave, u32 lane)
    {
        sums = sums_;
        s0 = 0;
        const u32 thread = wave * kWave + lane, row = thread / 8;
        chunk = thread & 7;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) {
            const u32 at = row + WAVES * 8 * i, o = output_of(at);
            p[i] = base + (second_of(at) ? second : 0) + (o < width ? o : 0u) * ld;
        }
        to = row * 128 + ((chunk ^ (row >> 1 & 7)) * 16);
        read = (lane & 15) * 128 + (((lane >> 4) ^ (lane >> 1 & 7)) * 16);
        request();
    }
    __device__ __forceinline__ void request()
    {
        const u32 s = s0 + chunk * 8, at = s + 8 <= sums ? s : sums - 8;
#pragma unroll
        for (u32 i = 0; i < kLoads; ++i) v[i] = load_any<u32x4>(p[i] + at);
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

// eight outputs and more
template <u32 W, u32 WAVES> struct BothAcrossAny {
    static constexpr bool kDirect = false;
    static constexpr u32 kLoads = W / 8 / WAVES, kRows = WAVES * kWave * 8 / W;
    static_assert(kRows % 16 == 0, "rows of another turn are turned alike");
    const __bf16 *p;
    u64 ld;
    u32 left, row, d;
    u32x4 v[kLoads];
    u32 to, read;

    __device__ __forceinline__ void init(const __bf16 *base, u64 second, u64 ld_, u32 width, u32 sums, u32 wave, u32 lane)
    {
        const u32 thread = wave * kWave + lane, chunk = thread % (W / 8), o = output_of(chunk * 8);
        row = thread / (W / 8);
        ld = ld_;
        left = sums;
        // outputs behind the last one are anything: their results are not kept
        const int at = o + 8 <= width ? (int)o : (int)width - 8;
        d = (u32)((int)o - at);
        p = base + (second_of(chunk * 8) ? second : 0) + at;
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

// Four values a lane of outputs m and of the next 16: eight consecutive ones, as in grouped_wide.hip
__device__ __forceinline__ u32x4 eight_of(const float (&lo)[4], const float (&hi)[4])
{
    const u32x2 a = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[0], lo[1]), pack_bf16(hi[0], hi[1]), false, false);
    const u32x2 b = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[2], lo[3]), pack_bf16(hi[2], hi[3]), false, false);
    return u32x4{a[0], b[0], a[1], b[1]};
}
// and back
__device__ __forceinline__ void four_and_four(u32x4 v, u32x2 (&of)[2])
{
    const u32x2 a = __builtin_amdgcn_permlane16_swap(v[0], v[2], false, false), b = __builtin_amdgcn_permlane16_swap(v[1], v[3], false, false);
    of[0] = u32x2{a[0], b[0]};
    of[1] = u32x2{a[1], b[1]};
}
// at most eight values at p, `count` of them there
template <bool ALL, bool PAST> __device__ __forceinline__ void store_eight(__bf16 *p, u32x4 v, u32 count)
{
    if (ALL || count >= 8) {
        store_vector<PAST>(p, v);
        return;
    }
#pragma unroll
    for (u32 e = 0; e < 7; ++e)
        if (e < count) p[e] = __builtin_bit_cast(__bf16, (unsigned short)(v[e / 2] >> (16 * (e % 2))));
}
// sum over the 16 lanes of a row of lanes
__device__ __forceinline__ float sixteen_sum(float v)
{
    const auto add = [&](u32 o) { v += __uint_as_float(o); };
    add(wave_dpp<0xB1, 0xf>(0u, __float_as_uint(v)));
    add(wave_dpp<0x4E, 0xf>(0u, __float_as_uint(v)));
    add(wave_dpp<0x141, 0xf>(0u, __float_as_uint(v)));
    add(wave_dpp<0x140, 0xf>(0u, __float_as_uint(v)));
    return v;
}

// LDS behind the operands: the tile's bias, and sums over its rows by the wavefronts beside each other
template <class S, u32 TP, u32 WP> constexpr u32 gated_lds() { return S::kLds + TP * 4 + S::kWaves / WP * TP * 4; }

// A workgroup takes tiles one after the other; as in grouped_linear4.hip the next one's first loads are on their way before this one's results
// leave, where operands go to LDS directly.
template <class S, u32 TP, u32 TQ, u32 WP, bool ACROSS, bool ANY, bool BACKWARD>
__global__ __launch_bounds__(S::kThreads, 2) void gated_wide_kernel(const GatedArgs r)
{
    extern __shared__ __align__(16) char wide_lds[];
    constexpr u32 kOut = TP / 2, kAcross = S::kWaves / WP, kPairs = S::kP / 4, kStores = kPairs * S::kQ * (BACKWARD ? 2 : 1);
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 p0 = wave % WP * (S::kP * 16), q0 = wave / WP * (S::kQ * 16);
    const u32 steps = (r.k + kStep - 1) / kStep;
    lds_char *lds = (lds_char *)wide_lds, *lb = lds + S::kLds;
    float *sums = reinterpret_cast<float *>(wide_lds + S::kLds + TP * 4);          // [wavefront across the rows][projection][output]

    // the tile: block ~0u for rows of no block
    struct Tile {
        u32 block, row0, height, begin, end, local, col0, width;
    };
    // the next one from number `id` on that there is
    const auto locate = [&](u32 &id, Tile &to) {
        for (; id < r.tiles; id += gridDim.x) {
            const u32 tile = tile_of_workgroup(id, r.tiles, S::kResident * kUnits);
            // four rows of tiles beside each other: what a die works on at once is four by eight of them, and shares most of its operands
            const u32 band = tile / (4 * r.col_tiles), in = tile - band * 4 * r.col_tiles, row_tile = 4 * band + in % 4;
            const RowRun run = find_run(r.offsets, r.blocks, r.rows, TQ, row_tile);
            if (!run.found) continue;
            to.block = uniform(run.block);
            to.begin = uniform(run.begin);
            to.end = uniform(run.end);
            to.local = uniform(run.local);
            to.row0 = uniform(run.begin + run.local * TQ);
            to.height = uniform(run.end - to.row0 < TQ ? run.end - to.row0 : TQ);
            to.col0 = uniform(in / 4 * kOut);
            to.width = uniform(r.n - to.col0 < kOut ? r.n - to.col0 : kOut);
            return true;
        }
        return false;
    };
    using Q = typename std::conditional<ANY, AlongAny<TQ, S::kWaves>, Along16<TQ, S::kWaves>>::type;
    using P = typename std::conditional<ACROSS, typename std::conditional<ANY, BothAcrossAny<TP, S::kWaves>, BothAcross16<TP, S::kWaves>>::type,
                                        typename std::conditional<ANY, BothAlongAny<TP, S::kWaves>, BothAlong16<TP, S::kWaves>>::type>::type;
    P p;
    Q q;
    const auto begin = [&](const Tile &t) {
        if (t.block == ~0u) return;
        const u32 at = afresh(lane);
        if (wave < TP / kWave) {
            const u32 h = wave * kWave / kOut, o = wave * kWave % kOut;
            const u64 from = r.bias ? reinterpret_cast<u64>(r.bias + (u64)t.block * 2 * r.n + h * r.n + t.col0) : reinterpret_cast<u64>(r.offsets);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer_of(reinterpret_cast<const void *>(from), r.bias ? t.width * 4 : 0u), lb + wave * kWave * 4, 4,
                                                     (int)((o + at) * 4), 0, 0, 0);
        }
        q.init(static_cast<const __bf16 *>(r.x) + (u64)t.row0 * r.ldx, r.ldx, t.height, r.k, wave, at);
        const __bf16 *w = static_cast<const __bf16 *>(r.w) + (u64)t.block * r.w_block;
        if constexpr (ACROSS) p.init(w + t.col0, r.n, r.ldw, t.width, r.k, wave, at);
        else p.init(w + (u64)t.col0 * r.ldw, (u64)r.n * r.ldw, r.ldw, t.width, r.k, wave, at);
#pragma unroll
        for (u32 part = 0; part < 2; ++part) {
            p.fill(lds + part * S::kPartP, wave);
            q.fill(lds + 2 * S::kPartP + part * S::kPartQ, wave);
        }
    };

    u32 id = blockIdx.x;
    Tile tile;
    if (!locate(id, tile)) return;
    wavefronts_meet<0x070>();               // nothing but those loads is on its way, here as for every other tile
    begin(tile);
    bool counted = false;
    for (;;) {
        if (counted) wavefronts_meet<(kStores & 15) | (kStores >> 4) << 14 | 0x070>();
        else wavefronts_meet<0x070>();
        // the sums begin with the bias; accumulators 2 m and 2 m + 1: outputs p0 / 2 + 16 m + 4 (lane / 16) and on, of the gate and of the other projection
        f32x4 acc[S::kP][S::kQ];
        const lds_char *own_bias = lb + (p0 / 2 + 4 * (afresh(lane) >> 4)) * 4;
#pragma unroll
        for (u32 i = 0; i < S::kP; ++i) {
            const f32x4 b = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(own_bias + (i % 2 * kOut + i / 2 * 16) * 4);
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j) acc[i][j] = tile.block != ~0u ? b : f32x4{};
        }
        if (tile.block != ~0u)
            wide_product<S, true>(p, q, steps, lds, wave, p0, q0, acc, [](const bf16x8 (&)[S::kQ]) {}, [](u32, const lds_char *) {});

        const Tile done = tile;
        const bool whole = done.height == TQ && done.width == kOut, inside = done.block != ~0u;
        const u32 at = afresh(lane), group = at >> 4;               // where its results go is not held through the product
        // outputs and row of a lane after the exchange of eight_of
        const auto out_of = [&](u32 m) { return p0 / 2 + 16 * (m + (group & 1)) + 8 * (group >> 1); };
        const auto row_of = [&](u32 j) { return q0 + 16 * j + (at & 15); };
        // dy, eight values a lane as results leave, kAhead of them on their way: number i is of outputs 2 (i / kQ) and rows i % kQ.  More of them cost
        // registers that the large tile has not (65 536 rows of 1024 -> 2048 in 32 blocks: three 764 us, one 717).
        constexpr u32 kAhead = 1;
        u32x4 up[kAhead];
        const __bf16 *dy_tile = static_cast<const __bf16 *>(r.dy) + (u64)done.row0 * r.lddy + done.col0;
        const auto fetch = [&](u32 i) {
            if (!BACKWARD || i >= kPairs * S::kQ) return;
            const u32 o = out_of(2 * (i / S::kQ)), row = row_of(i % S::kQ);
            u32x4 v = {0, 0, 0, 0};
            if (inside && row < done.height) {
                const __bf16 *from = dy_tile + (u64)row * r.lddy + o;
                if (o + 8 <= done.width) {
                    v = load_any<u32x4>(from);
                } else if (ANY) {
#pragma unroll
                    for (u32 e = 0; e < 7; ++e)
                        if (o + e < done.width) v[e / 2] |= (u32)__builtin_bit_cast(unsigned short, from[e]) << (16 * (e % 2));
                }
            }
            up[i % kAhead] = v;
        };
#pragma unroll
        for (u32 i = 0; i < kAhead; ++i) fetch(i);
        id += gridDim.x;
        const bool more = locate(id, tile);
        // nothing may be on its way into LDS when it is filled for the next tile, or when the workgroup ends
        wavefronts_meet<0x070>();
        if (!ANY && more) begin(tile);
        asm volatile("" ::: "memory");                              // the stores stay behind those loads
        __bf16 *out = static_cast<__bf16 *>(r.out) + (u64)done.row0 * r.ldo + done.col0;
        const auto finish = [&](auto act, auto all) {
            constexpr bool kEight = !ANY || all, kPast = !BACKWARD && all;
            if constexpr (!ANY && all) stores_begin<kStores>();
#pragma unroll
            for (u32 m = 0; m < 2 * kPairs; m += 2) {
                float sum[2][2][4] = {};                            // [of m, m + 1][projection]
                const u32 o = out_of(m);
#pragma unroll
                for (u32 j = 0; j < S::kQ; ++j) {
                    const u32 row = row_of(j);
                    __bf16 *to = out + (u64)row * r.ldo + o;
                    const bool there = all || (row < done.height && o < done.width);
                    if constexpr (!BACKWARD) {
                        float y[2][4];
#pragma unroll
                        for (u32 h = 0; h < 2; ++h)
#pragma unroll
                            for (u32 v = 0; v < 4; ++v) y[h][v] = gated(act, acc[2 * (m + h)][j][v], acc[2 * (m + h) + 1][j][v]);
                        const u32x4 v = eight_of(y[0], y[1]);
                        if (there) store_eight<kEight, kPast>(to, v, done.width - o);
                    } else {
                        float da[2][4], du[2][4];
                        u32x2 dy[2];
                        four_and_four(up[(m / 2 * S::kQ + j) % kAhead], dy);
                        fetch(m / 2 * S::kQ + j + kAhead);
#pragma unroll
                        for (u32 h = 0; h < 2; ++h)
#pragma unroll
                            for (u32 v = 0; v < 4; ++v) {
                                const float g = __uint_as_float(v % 2 ? dy[h][v / 2] & 0xffff0000u : dy[h][v / 2] << 16);
                                gated_gradient(act, acc[2 * (m + h)][j][v], acc[2 * (m + h) + 1][j][v], g, da[h][v], du[h][v]);
                                // what is not there has a dy of 0, but may be multiplied by what is not finite
                                const bool on = all || (row < done.height && p0 / 2 + 16 * (m + h) + 4 * group + v < done.width);
                                da[h][v] = on ? da[h][v] : 0.0f;
                                du[h][v] = on ? du[h][v] : 0.0f;
                                sum[h][0][v] += da[h][v];
                                sum[h][1][v] += du[h][v];
                            }
                        const u32x4 va = eight_of(da[0], da[1]), vu = eight_of(du[0], du[1]);
                        if (there) {
                            store_eight<kEight, kPast>(to, va, done.width - o);
                            store_eight<kEight, kPast>(to + r.n, vu, done.width - o);
                        }
                    }
                }
                if (BACKWARD && r.part) {
#pragma unroll
                    for (u32 h = 0; h < 2; ++h)
#pragma unroll
                        for (u32 s = 0; s < 2; ++s)
#pragma unroll
                            for (u32 v = 0; v < 4; ++v) {
                                const float over_rows = sixteen_sum(sum[h][s][v]);
                                if ((at & 15) == 0) sums[(wave / WP * 2 + s) * kOut + p0 / 2 + 16 * (m + h) + 4 * group + v] = over_rows;
                            }
                }
            }
            if constexpr (!ANY && all) stores_end();
        };
        // Tiles of which everything is there, and the others.  The gradients are read again at once, and not stored past the caches.  (A third form
        // of y's, for whole tiles that go through the caches, costs the others 3 %: 414 us, with it 423.)
        counted = !ANY && whole && inside && (BACKWARD || r.past);
        const auto finish_act = [&](auto act) {
            if (whole && (BACKWARD || r.past)) finish(act, std::true_type{});
            else finish(act, std::false_type{});
        };
        // rows of no block get zeros: the activation of 0 is 0, and so is what a dy of 0 is multiplied by
        if (inside && r.act == LMK_GS_SILU) finish_act(std::integral_constant<u32, LMK_GS_SILU>{});
        else if (inside && r.act == LMK_GS_GELU) finish_act(std::integral_constant<u32, LMK_GS_GELU>{});
        else finish_act(std::integral_constant<u32, LMK_GS_RELU>{});
        if (BACKWARD && r.part) {
            wavefronts_meet<0xC07F>();                              // LDS alone is waited for
            if (inside) {
                RowRun run;
                run.block = done.block;
                run.begin = done.begin;
                run.end = done.end;
                run.local = done.local;
                for (u32 i = threadIdx.x; i < 2 * kOut; i += S::kThreads) {
                    const u32 s = i / kOut, o = i % kOut;
                    if (o >= done.width) continue;
                    float over_rows = 0.0f;
#pragma unroll
                    for (u32 w = 0; w < kAcross; ++w) over_rows += sums[(w * 2 + s) * kOut + o];
                    set_of(r, run, TQ)[s * r.n + done.col0 + o] = over_rows;
                }
            }
        }
        if (!more) return;
        if (ANY) begin(tile);
    }
}

bool sixteen(const void *p, u64 ld) { return ld % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0; }

bool gated_sixteen(const GatedArgs &r)
{
    return r.k % 8 == 0 && r.n % 8 == 0 && sixteen(r.x, r.ldx) && sixteen(r.w, r.ldw) && r.w_block % 8 == 0;
}

// As large_tiles in grouped_wide.hip, with both projections' outputs.  256 x 256 / 128 x 128, y of 1024 -> 512 in 8 blocks: 4096 rows 27 / 17 us,
// 65 536 121 / 145; 16 384 rows of 2048 -> 4096 in 4 413 / 490.
bool large_tiles(const GatedArgs &r)
{
    const auto share = [&](u32 side) { return __builtin_ceilf((float)r.rows / side + 0.5f * (r.blocks - 1)) * ((2 * r.n + side - 1) / side); };
    return gated_sixteen(r) && __builtin_ceilf(share(256) / 256) < 0.7f * share(128) / 512;
}

template <u32 TP, u32 TQ, u32 WP, u32 WQ, bool ACROSS, bool ANY, bool BACKWARD>
hipError_t wide_go(GatedArgs r, hipStream_t stream)
{
    using S = Shape<TP, TQ, WP, WQ>;
    constexpr u32 lds = gated_lds<S, TP, WP>(), at_once = 8 * kUnits * S::kResident;
    r.past = !BACKWARD && past_caches(r.out, r.ldo * 2, (u64)r.rows * r.n * 2);
    r.col_tiles = (r.n + TP / 2 - 1) / (TP / 2);
    r.tiles = (u32)((max_runs(r.rows, r.blocks, TQ) + 3) / 4 * 4 * r.col_tiles);
    auto kernel = gated_wide_kernel<S, TP, TQ, WP, ACROSS, ANY, BACKWARD>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(r.tiles < at_once ? r.tiles : at_once), dim3(S::kThreads), lds, stream, r);
    return hipGetLastError();
}
template <bool ACROSS, bool BACKWARD>
hipError_t wide_shape(const GatedArgs &r, hipStream_t stream)
{
    if (!gated_sixteen(r)) return wide_go<128, 128, 2, 2, ACROSS, true, BACKWARD>(r, stream);
    if (large_tiles(r)) return wide_go<256, 256, 2, 4, ACROSS, false, BACKWARD>(r, stream);
    return wide_go<128, 128, 2, 2, ACROSS, false, BACKWARD>(r, stream);
}

}  // namespace

// Offsets inside a tile are 32 bits wide.  Narrower than eight: the general kernel.
bool gated_wide_fits(const GatedArgs &r)
{
    constexpr u64 most = 1u << 21;
    return r.k >= 8 && r.n >= 8 && r.ldx <= most && r.ldw <= most;
}

u32 gated_wide_rows(const GatedArgs &r) { return large_tiles(r) ? 256 : 128; }

u64 gated_wide_threads(const GatedArgs &r)
{
    const u32 side = gated_wide_rows(r);
    return (max_runs(r.rows, r.blocks, side) + 3) * ((r.n + side / 2 - 1) / (side / 2)) * (side * 2);
}

hipError_t launch_gated_wide(const GatedArgs &r, hipStream_t stream)
{
    if (r.in_major) return r.dy ? wide_shape<true, true>(r, stream) : wide_shape<true, false>(r, stream);
    return r.dy ? wide_shape<false, true>(r, stream) : wide_shape<false, false>(r, stream);
}

}  // namespace lmk
