// All gradients of a grouped layer of small matrices (the decoder's: 35 x 96, 32 x 70) in one pass: dy and x are read once,
// dx leaves once, and the sums over rows stay in registers.  As in the forward kernel a workgroup keeps its block's
// matrix in LDS and its four wavefronts walk through a run of the block's rows in tiles of 16, each by itself:
//     dx = dy w_g     weights on the matrix instruction's rows, dy's rows on its columns
//     dw += x^T dy    inputs on its rows, outputs on its columns, summed over the tile's 16 rows
// (v_mfma_f32_16x16x4_f32).  Of both, a tile of dy and of x (widened from its 8-bit form) is the operand, read from LDS.
// db is added up from the values of dy on their way to the second product.  At the end the four wavefronts' sums meet in LDS
// and are added in their order.
//
// 300 000 rows in 24 blocks: 35 x 96 in 86 us, 32 x 70 with the gate in 57 us.  Bound by the float32 instructions (35 us for the
// first at their rate), which wait for the LDS reads in front of them: the sums of 96 x 48 leave registers for two
// wavefronts a SIMD.  About 13 us are a run's own costs: weights into LDS, the four wavefronts' sums joined.
#include "grouped_narrow.h"

namespace lmk {

namespace {

// The same from the 8-bit form, widened on the way into LDS
template <u32 N> struct CodePieces {
    Turns t;
    u32 next[N], scale[N];
    u32 kp, turn_floats, rows;

    __device__ __forceinline__ void init(u32 kp_, u32 width, u32 lane)
    {
        t.init(width, lane);
        kp = kp_;
        turn_floats = t.rows * pitch_of(width);
    }
    __device__ __forceinline__ void request(const char *codes, const uint8_t *scales, u32 rows_)
    {
        rows = rows_;
        if (rows == 0) return;
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            const u32 row = t.row + i * t.rows, at = (t.row < rows && row < rows ? row : 0u) * kp + t.col;
            next[i] = *reinterpret_cast<const u32 *>(codes + at);
            scale[i] = scales[at / 32];
        }
    }
    __device__ __forceinline__ void put(float *lds) const
    {
#pragma unroll
        for (u32 i = 0; i < N; ++i) {
            const u32 row = t.row + i * t.rows;
            // the byte 0 makes zeros of any codes
            const float step = step_of(row < rows ? scale[i] : 0u);
            if (t.row < kTileRows && row < kTileRows)
                *reinterpret_cast<f32x4 *>(lds + t.to + i * turn_floats) =
                    f32x4{value_of(next[i], 0, step), value_of(next[i], 1, step), value_of(next[i], 2, step), value_of(next[i], 3, step)};
        }
    }
};

constexpr u32 kFillers = 64;            // workgroups for dx of rows of no block

// Steps of dx's product, four outputs each, in whole turns of four.  Those behind the last output have zeros on both sides: a
// weight that is not finite, multiplied by a zero of dy, would be a NaN.
__host__ __device__ constexpr u32 whole_steps(u32 n) { return (n + 15) / 16 * 4; }

// floats between the outputs of the joined sums in LDS
constexpr u32 sums_pitch(u32 ck) { return 16 * ck + 4; }
constexpr u32 sums_floats(u32 cn, u32 ck) { return 16 * cn * sums_pitch(ck) + 16 * cn; }

// LDS of the widest matrices of a shape: weights and the four wavefronts' tiles, then their sums in the same place
constexpr u32 shape_lds(u32 cn, u32 ck)
{
    const u32 before = 4 * cn * ck * kWave + 4 * kTileRows * (pitch_of(16 * cn) + pitch_of(16 * ck)), sums = 4 * sums_floats(cn, ck);
    return (before > sums ? before : sums) * 4;
}
// Workgroups of a compute unit (wavefronts of a SIMD), what the registers of the sums and LDS both leave: three up to twelve tiles
// of sums, whose wavefronts take at most 168 registers, two up to 24.  LDS is given out in pieces of 1280 bytes; 64 x 48 and 96 x 32
// have two workgroups for it, 80 x 64 and 96 x 64 one.
constexpr u32 resident(u32 cn, u32 ck)
{
    const u32 registers = cn * ck <= 12 ? 3 : 2, lds = kLdsBytes / ((shape_lds(cn, ck) + kLdsPiece - 1) / kLdsPiece * kLdsPiece);
    return registers < lds ? registers : lds;
}

// CN, CK: 16 outputs and 16 inputs each
template <u32 CN, u32 CK, bool CODES>
__global__ __launch_bounds__(256, resident(CN, CK)) void narrow_backward_kernel(const BackwardArgs r)
{
    extern __shared__ __align__(16) float narrow_lds[];
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    if (blockIdx.x >= r.runs) {
        // rows in front of the first block and behind the last one
        u32 front = r.offsets[0], back = r.offsets[r.blocks];
        front = front < r.rows ? front : r.rows;
        back = back < front ? front : back < r.rows ? back : r.rows;
        const u32 count = front + (r.rows - back);
        for (u32 i = blockIdx.x - r.runs; i < count && r.dx; i += kFillers)
            for (u32 c = threadIdx.x; c < r.k; c += 256) r.dx[(u64)(i < front ? i : back + (i - front)) * r.lddx + c] = 0.0f;
        return;
    }
    const u32 pn = pitch_of(r.n), pk = pitch_of(r.k), kp = (r.k + 31) / 32 * 32, steps = (r.n + 3) / 4;
    float *lw = narrow_lds, *ly = lw + r.shared + wave * kTileRows * (pn + pk), *lx = ly + kTileRows * pn;
    BlockRun run;
    if (!run.find(r.offsets, r.blocks, r.rows, r.per, blockIdx.x)) return;
    const u32 row0 = run.row, height = run.count, lane = threadIdx.x & (kWave - 1), j = lane & 15, q = lane >> 4;
    if (r.dx) {
        stage_weights<float, CK>(lw, r.w + (u64)run.block * r.w_block, r.ldw, r.in_major == 0, r.n, r.k);
        for (u32 i = steps * CK * kWave + threadIdx.x; i < whole_steps(r.n) * CK * kWave; i += 256) lw[i] = 0.0f;
    }
    __syncthreads();

    const u32 tiles = (height + kTileRows - 1) / kTileRows;
    const char *dy = reinterpret_cast<const char *>(r.dy + (u64)row0 * r.lddy);
    const char *x = static_cast<const char *>(r.x) + (u64)row0 * (CODES ? kp : r.ldx * 4);
    const uint8_t *scale = r.scale + (u64)row0 * (kp / 32);
    Pieces<float, turns_of(4 * CN)> tile_y;
    tile_y.init(r.lddy, r.n, lane);
    typename std::conditional<CODES, CodePieces<turns_of(4 * CK)>, Pieces<float, turns_of(4 * CK)>>::type tile_x;
    if constexpr (CODES) tile_x.init(kp, r.k, lane);
    else tile_x.init(r.ldx, r.k, lane);
    clear_gaps(ly, r.n, lane);
    clear_gaps(lx, r.k, lane);
    auto request = [&](u32 tile) {
        const u32 rows = tile < tiles ? height - tile * kTileRows : 0u;
        const u64 first = (u64)tile * kTileRows;
        tile_y.request(dy + first * r.lddy * 4, rows);
        if constexpr (CODES) tile_x.request(x + first * kp, scale + first * (kp / 32), r.x ? rows : 0u);
        else tile_x.request(x + first * r.ldx * 4, r.x ? rows : 0u);
    };
    f32x4 dw[CK][CN] = {};
    float db[CN] = {};
    auto put = [&]() {
        tile_y.put(ly);
        tile_x.put(lx);
    };
    request(wave);
    put();
    request(wave + 4);
    for (u32 tile = wave; tile < tiles; tile += 4) {
        const u32 base = tile * kTileRows, left = height - base;
        wave_meets();
        // sums over the tile's rows; columns that are not there hold what lies behind a row, and reach only results that are not kept
        float fy[2][CN], fx[2][CK];
        auto operands = [&](u32 s, u32 at) {
#pragma unroll
            for (u32 b = 0; b < CN; ++b) fy[at][b] = 16 * b + j < pn ? ly[(4 * s + q) * pn + 16 * b + j] : 0.0f;
#pragma unroll
            for (u32 a = 0; a < CK; ++a) fx[at][a] = 16 * a + j < pk ? lx[(4 * s + q) * pk + 16 * a + j] : 0.0f;
        };
        operands(0, 0);
#pragma unroll
        for (u32 s = 0; s < 4; ++s) {
            if (s < 3) operands(s + 1, (s + 1) & 1);
#pragma unroll
            for (u32 b = 0; b < CN; ++b) db[b] += fy[s & 1][b];
#pragma unroll
            for (u32 a = 0; a < CK; ++a)
#pragma unroll
                for (u32 b = 0; b < CN; ++b) dw[a][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fx[s & 1][a], fy[s & 1][b], dw[a][b], 0, 0, 0);
        }
        f32x4 acc[CK] = {};
        if (r.dx) {
            // two steps' operands are on their way from LDS while two are multiplied; behind the last one zeros.  Behind the last whole
            // turn: what lies there in LDS, and is not multiplied
            float v[2][2], w[2][2][CK];
            auto fetch = [&](u32 s, u32 at) {
#pragma unroll
                for (u32 e = 0; e < 2; ++e) {
                    const float y = ly[j * pn + 4 * (s + e) + q];
                    v[at][e] = s + e < steps ? y : 0.0f;
#pragma unroll
                    for (u32 c = 0; c < CK; ++c) w[at][e][c] = lw[((s + e) * CK + c) * kWave + lane];
                }
            };
            auto multiply = [&](u32 at) {
#pragma unroll
                for (u32 e = 0; e < 2; ++e)
#pragma unroll
                    for (u32 c = 0; c < CK; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[at][e][c], v[at][e], acc[c], 0, 0, 0);
            };
            fetch(0, 0);
            for (u32 s = 0; s < steps; s += 4) {
                fetch(s + 2, 1);
                multiply(0);
                fetch(s + 4, 0);
                multiply(1);
            }
            if (r.gate) {
#pragma unroll
                for (u32 c = 0; c < CK; ++c) {
                    if (16 * c + 4 * q >= r.k) continue;
                    const f32x4 g = *reinterpret_cast<const f32x4 *>(lx + j * pk + 16 * c + 4 * q);
#pragma unroll
                    for (u32 e = 0; e < 4; ++e) acc[c][e] = g[e] <= 0.0f ? 0.0f : acc[c][e];          // NaN lets pass
                }
            }
        }
        // The next tile takes this one's place before the results leave: what is waited for there is then this tile's loads and
        // not its stores.
        wave_meets();
        put();
        request(tile + 8);
        if (r.dx && j < left) {
            float *out = r.dx + (u64)(row0 + base) * r.lddx + j * (u32)r.lddx;
#pragma unroll
            for (u32 c = 0; c < CK; ++c) {
                const u32 col = 16 * c + 4 * q;
                if (col + 4 <= r.k) {
                    store4(out + col, acc[c]);
                } else {
#pragma unroll
                    for (u32 e = 0; e < 3; ++e)
                        if (col + e < r.k) out[col + e] = acc[c][e];
                }
            }
        }
    }
    // ---- the four wavefronts' sums, [output][input] and then db each
    constexpr u32 ps = sums_pitch(CK), part = sums_floats(CN, CK);
    __syncthreads();
    float *ls = narrow_lds + wave * part, *lb = ls + 16 * CN * ps;
#pragma unroll
    for (u32 b = 0; b < CN; ++b) {
        db[b] += __shfl_xor(db[b], 16, kWave);
        db[b] += __shfl_xor(db[b], 32, kWave);
#pragma unroll
        for (u32 a = 0; a < CK; ++a) *reinterpret_cast<f32x4 *>(ls + (16 * b + j) * ps + 16 * a + 4 * q) = dw[a][b];
        if (q == 0) lb[16 * b + j] = db[b];
    }
    __syncthreads();
    const u32 size = r.n * r.k;
    float *to_w = run.whole ? r.dw + (u64)run.block * size : r.part + (u64)run.partial() * (size + r.n);
    float *to_b = run.whole ? r.db + (u64)run.block * r.n : r.part + (u64)run.partial() * (size + r.n) + size;
    const auto joined = [&](u32 at) { return ((narrow_lds[at] + narrow_lds[part + at]) + narrow_lds[2 * part + at]) + narrow_lds[3 * part + at]; };
    if (r.dw) {
        const u32 width = r.in_major ? r.n : r.k;
#pragma unroll 4
        for (u32 i = threadIdx.x; i < size; i += 256) {
            const u32 outer = i / width, inner = i - outer * width;
            to_w[i] = joined(r.in_major ? inner * ps + outer : outer * ps + inner);
        }
    }
    if (r.db)
        for (u32 i = threadIdx.x; i < r.n; i += 256) to_b[i] = joined(16 * CN * ps + i);
}

template <u32 CN, u32 CK>
hipError_t narrow_backward_go(BackwardArgs r, bool codes, hipStream_t stream)
{
    const u32 weights = whole_steps(r.n) * CK * kWave, sums = 4 * sums_floats(CN, CK);
    const u32 tiles = 4 * kTileRows * (pitch_of(r.n) + pitch_of(r.k));
    r.shared = weights;
    const u32 lds = (weights + tiles > sums ? weights + tiles : sums) * 4;
    auto kernel = codes ? narrow_backward_kernel<CN, CK, true> : narrow_backward_kernel<CN, CK, false>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(r.runs + kFillers), dim3(256), lds, stream, r);
    return hipGetLastError();
}
template <u32 CN>
hipError_t narrow_backward_k(const BackwardArgs &r, bool codes, hipStream_t stream)
{
    switch ((r.k + 15) / 16) {
    case 1: return narrow_backward_go<CN, 1>(r, codes, stream);
    case 2: return narrow_backward_go<CN, 2>(r, codes, stream);
    case 3: return narrow_backward_go<CN, 3>(r, codes, stream);
    default: return narrow_backward_go<CN, 4>(r, codes, stream);
    }
}

}  // namespace

bool narrow_backward_fits(const BackwardArgs &r, bool codes)
{
    if (r.n < 4 || r.k < 4 || r.n > 96 || r.k > 64) return false;
    return r.lddy <= kNarrowStride && r.lddx <= kNarrowStride && (codes || r.ldx <= kNarrowStride);
}

// outputs in tiles of 16, as the kernels are built for them
static u32 out_tiles(u32 n) { return n <= 32 ? 2 : n <= 64 ? 4 : n <= 80 ? 5 : 6; }

u32 narrow_backward_slots(u32 n, u32 k) { return 256 * resident(out_tiles(n), (k + 15) / 16); }

hipError_t launch_narrow_backward(const BackwardArgs &r, bool codes, hipStream_t stream)
{
    switch (out_tiles(r.n)) {
    case 2: return narrow_backward_k<2>(r, codes, stream);
    case 4: return narrow_backward_k<4>(r, codes, stream);
    case 5: return narrow_backward_k<5>(r, codes, stream);
    default: return narrow_backward_k<6>(r, codes, stream);
    }
}

}  // namespace lmk
