// Gated layers in bfloat16 on the bfloat16 matrix instructions: the tiles of grouped_wide.hip, of whose rows of weights 16 are of the
// gate and the next 16 of the other projection, in turns.  A lane then has both projections of the same four outputs in neighbouring
// accumulators, and the activation, the product and their gradients need no exchange.
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
// at most eight values at p, `count` of them there
template <bool ANY> __device__ __forceinline__ void store_eight(__bf16 *p, u32x4 v, u32 count)
{
    if (!ANY || count >= 8) {
        store_any(p, v);
        return;
    }
#pragma unroll
    for (u32 e = 0; e < 8; ++e)
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

template <class S, u32 TP, u32 TQ, u32 WP, bool ACROSS, bool ANY, bool BACKWARD>
__global__ __launch_bounds__(S::kThreads, 2) void gated_wide_kernel(const GatedArgs r)
{
    extern __shared__ __align__(16) char wide_lds[];
    constexpr u32 kOut = TP / 2;
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, S::kResident * kUnits);
    const u32 row_tile = tile / r.col_tiles, col0 = (tile - row_tile * r.col_tiles) * kOut;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, TQ, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * TQ;
    const u32 height = run.end - row0 < TQ ? run.end - row0 : TQ;
    const u32 width = r.n - col0 < kOut ? r.n - col0 : kOut;
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 p0 = wave % WP * (S::kP * 16), q0 = wave / WP * (S::kQ * 16);
    const bool inside = run.block != ~0u;
    lds_char *lds = (lds_char *)wide_lds;
    f32x4 acc[S::kP][S::kQ] = {};
    if (inside) {
        const u32 steps = (r.k + kStep - 1) / kStep;
        const auto nothing = [](const bf16x8 (&)[S::kQ]) {};
        const auto unseen = [](u32, const lds_char *) {};
        typename std::conditional<ANY, AlongAny<TQ, S::kWaves>, Along16<TQ, S::kWaves>>::type q;
        q.init(static_cast<const __bf16 *>(r.x) + (u64)row0 * r.ldx, r.ldx, height, r.k, wave, lane);
        const __bf16 *w = static_cast<const __bf16 *>(r.w) + (u64)run.block * r.w_block;
        if constexpr (ACROSS) {
            typename std::conditional<ANY, BothAcrossAny<TP, S::kWaves>, BothAcross16<TP, S::kWaves>>::type p;
            p.init(w + col0, r.n, r.ldw, width, r.k, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, nothing, unseen);
        } else {
            typename std::conditional<ANY, BothAlongAny<TP, S::kWaves>, BothAlong16<TP, S::kWaves>>::type p;
            p.init(w + (u64)col0 * r.ldw, (u64)r.n * r.ldw, r.ldw, width, r.k, wave, lane);
            wide_product<S>(p, q, steps, lds, wave, p0, q0, acc, nothing, unseen);
        }
    }
    // accumulators 2 m and 2 m + 1: outputs p0 / 2 + 16 m + 4 group and on, of the gate and of the other projection
    const u32 group = lane >> 4;
    __bf16 *out = static_cast<__bf16 *>(r.out) + (u64)row0 * r.ldo + col0;
    const float *bias = r.bias && inside ? r.bias + (u64)run.block * 2 * r.n + col0 : nullptr;
    float *sums = reinterpret_cast<float *>(wide_lds);          // BACKWARD: [wavefront across the rows][2][outputs]
    if (BACKWARD && r.part) __syncthreads();                    // the product is out of LDS
#pragma unroll
    for (u32 m = 0; m < S::kP / 2; m += 2) {
        f32x4 b[2][2] = {};                                     // [of m, m + 1][projection]
        float sum[2][2][4] = {};
        if (bias) {
#pragma unroll
            for (u32 h = 0; h < 2; ++h)
#pragma unroll
                for (u32 v = 0; v < 4; ++v) {
                    const u32 o = p0 / 2 + 16 * (m + h) + 4 * group + v;
                    b[h][0][v] = o < width ? bias[o] : 0.0f;
                    b[h][1][v] = o < width ? bias[r.n + o] : 0.0f;
                }
        }
        const u32 o = p0 / 2 + 16 * (m + (group & 1)) + 8 * (group >> 1);           // after the exchange
#pragma unroll
        for (u32 j = 0; j < S::kQ; ++j) {
            const u32 row = q0 + 16 * j + (lane & 15);
            if constexpr (!BACKWARD) {
                float y[2][4];
#pragma unroll
                for (u32 h = 0; h < 2; ++h)
#pragma unroll
                    for (u32 v = 0; v < 4; ++v)
                        y[h][v] = gated(r.act, acc[2 * (m + h)][j][v] + b[h][0][v], acc[2 * (m + h) + 1][j][v] + b[h][1][v]);
                u32x4 v = eight_of(y[0], y[1]);
                if (!inside) v = u32x4{0, 0, 0, 0};
                if (row < height && o < width) store_eight<ANY>(out + (u64)row * r.ldo + o, v, width - o);
            } else {
                float da[2][4], du[2][4];
#pragma unroll
                for (u32 h = 0; h < 2; ++h) {
                    const u32 at = p0 / 2 + 16 * (m + h) + 4 * group;
                    const bool on = inside && row < height && at < width;
                    f32x4 dy = {0.0f, 0.0f, 0.0f, 0.0f};
                    const __bf16 *from = static_cast<const __bf16 *>(r.dy) + (u64)(row0 + row) * r.lddy + col0 + at;
                    if (on && (!ANY || at + 4 <= width)) {
                        dy = load4(from);
                    } else if (ANY && on) {
#pragma unroll
                        for (u32 v = 0; v < 3; ++v)
                            if (at + v < width) dy[v] = (float)from[v];
                    }
#pragma unroll
                    for (u32 v = 0; v < 4; ++v) {
                        gated_gradient(r.act, acc[2 * (m + h)][j][v] + b[h][0][v], acc[2 * (m + h) + 1][j][v] + b[h][1][v], dy[v], da[h][v], du[h][v]);
                        const bool there = on && (!ANY || at + v < width);
                        da[h][v] = there ? da[h][v] : 0.0f;
                        du[h][v] = there ? du[h][v] : 0.0f;
                        sum[h][0][v] += da[h][v];
                        sum[h][1][v] += du[h][v];
                    }
                }
                const u32x4 va = eight_of(da[0], da[1]), vu = eight_of(du[0], du[1]);
                if (row < height && o < width) {
                    store_eight<ANY>(out + (u64)row * r.ldo + o, va, width - o);
                    store_eight<ANY>(out + (u64)row * r.ldo + r.n + o, vu, width - o);
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
                        const float all = sixteen_sum(sum[h][s][v]);
                        if ((lane & 15) == 0) sums[(wave / WP * 2 + s) * kOut + p0 / 2 + 16 * (m + h) + 4 * group + v] = all;
                    }
        }
    }
    if (BACKWARD && r.part) {
        __syncthreads();
        if (!inside) return;
        constexpr u32 kAcross = S::kWaves / WP;
        for (u32 i = threadIdx.x; i < 2 * kOut; i += S::kThreads) {
            const u32 s = i / kOut, o = i % kOut;
            if (o >= width) continue;
            float all = 0.0f;
#pragma unroll
            for (u32 q = 0; q < kAcross; ++q) all += sums[(q * 2 + s) * kOut + o];
            set_of(r, run, TQ)[s * r.n + col0 + o] = all;
        }
    }
}

bool sixteen(const void *p, u64 ld) { return ld % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0; }

bool gated_sixteen(const GatedArgs &r)
{
    return r.k % 8 == 0 && r.n % 8 == 0 && sixteen(r.x, r.ldx) && sixteen(r.w, r.ldw) && r.w_block % 8 == 0;
}

// as large_tiles in grouped_wide.hip, with both projections' outputs
bool large_tiles(const GatedArgs &r)
{
    const auto share = [&](u32 side) { return __builtin_ceilf((float)r.rows / side + 0.5f * (r.blocks - 1)) * ((2 * r.n + side - 1) / side); };
    return gated_sixteen(r) && __builtin_ceilf(share(256) / 256) < 0.7f * share(128) / 512;
}

template <u32 TP, u32 TQ, u32 WP, u32 WQ, bool ACROSS, bool ANY, bool BACKWARD>
hipError_t wide_go(GatedArgs r, hipStream_t stream)
{
    using S = Shape<TP, TQ, WP, WQ>;
    r.col_tiles = (r.n + TP / 2 - 1) / (TP / 2);
    r.tiles = (u32)(max_runs(r.rows, r.blocks, TQ) * r.col_tiles);
    auto kernel = gated_wide_kernel<S, TP, TQ, WP, ACROSS, ANY, BACKWARD>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(r.tiles), dim3(S::kThreads), S::kLds, stream, r);
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
    return max_runs(r.rows, r.blocks, side) * ((r.n + side / 2 - 1) / (side / 2)) * (side * 2);
}

hipError_t launch_gated_wide(const GatedArgs &r, hipStream_t stream)
{
    if (r.in_major) return r.dy ? wide_shape<true, true>(r, stream) : wide_shape<true, false>(r, stream);
    return r.dy ? wide_shape<false, true>(r, stream) : wide_shape<false, false>(r, stream);
}

}  // namespace lmk
