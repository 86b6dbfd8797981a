// Grouped layers whose weights are small (the decoder's: 35 x 96, 32 x 70): memory is all of it, so a row is read once and its
// results leave once.  A workgroup keeps its block's whole matrix in LDS, in the order the matrix instructions take it, and
// its four wavefronts walk through a run of the block's rows in tiles of 16, each by itself: the next tile's rows are
// on their way to registers while a tile is multiplied, and nothing is waited for in common.
//
// v_mfma_f32_16x16x4_f32 with the weights on its rows and the layer's rows on its columns: a lane has four
// consecutive outputs of a row, one 16-byte store.  In LDS a row of x takes a pitch of 4 (odd) floats: the 16 rows and
// four sum indices that an instruction reads are on 64 different banks.
//
// 300 000 rows in 24 blocks, with the 8-bit form of x written on the way: 35 x 96 in 50 us (177 MB, 3.5 TB/s), 32 x 70 in 36
// (132 MB, 3.7 TB/s); without it 35 x 96 in 38 us (157 MB, 4.1 TB/s).  What is left above a copy's 4.9 TB/s is the weights' way into LDS at the start of every run, and a wavefront's own
// chain of load, LDS, products and store, of which four to a SIMD hide most.
#include "grouped_narrow.h"

namespace lmk {

namespace {

// CT: tiles of 16 columns; PIECES: turns in which a wavefront brings a tile of x
// KEEP: also writes the 8-bit form of x; GATE: 0 none, 1 values, 2 codes
template <u32 CT, u32 PIECES, bool KEEP, u32 GATE>
__global__ __launch_bounds__(256, PIECES <= 4 ? 4 : 3) void narrow_rows_kernel(const RowsArgs r)
{
    extern __shared__ __align__(16) float narrow_lds[];
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, r.per, blockIdx.x);
    if (!run.found) return;
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), j = lane & 15, q = lane >> 4;
    const u32 row0 = run.begin + run.local * r.per;
    const u32 height = run.end - row0 < r.per ? run.end - row0 : r.per;
    const bool inside = run.block != ~0u;
    const u32 steps = (r.sums + 3) / 4, pitch = pitch_of(r.sums);
    float *lw = narrow_lds, *lb = lw + steps * CT * kWave, *lx = lb + CT * 16 + wave * kTileRows * pitch;

    if (inside) {
        stage_weights<float, CT>(lw, static_cast<const float *>(r.w) + (u64)run.block * r.w_block, r.ldw, r.across, r.sums, r.cols);
        for (u32 i = threadIdx.x; i < CT * 16; i += 256) lb[i] = r.bias && i < r.cols ? r.bias[(u64)run.block * r.cols + i] : 0.0f;
    }
    __syncthreads();

    const u32 tiles = (height + kTileRows - 1) / kTileRows;
    const char *x = reinterpret_cast<const char *>(static_cast<const float *>(r.a) + (u64)row0 * r.lda);
    Pieces<float, PIECES> tile_of_x;
    tile_of_x.init(r.lda, r.sums, lane);
    clear_gaps(lx, r.sums, lane);
    auto request = [&](u32 tile) {
        tile_of_x.request(x + (u64)tile * kTileRows * r.lda * sizeof(float), inside && tile < tiles ? height - tile * kTileRows : 0u);
    };
    request(wave);
    tile_of_x.put(lx);
    request(wave + 4);
    for (u32 tile = wave; tile < tiles; tile += 4) {
        const u32 base = tile * kTileRows, left = height - base;
        wave_meets();
        if constexpr (KEEP) {
            // eight values a lane, four lanes for those that share a step; rows of no block are the zeros that request() left
            const u32 m = lane / 4, eight = lane % 4, kp = (r.sums + 31) / 32 * 32;
            char *codes = reinterpret_cast<char *>(r.keep_codes) + (u64)(row0 + base) * kp + m * kp + 8 * eight;
            uint8_t *scales = r.keep_scale + (u64)(row0 + base) * (kp / 32) + m * (kp / 32);
            const float *row = lx + m * pitch + 8 * eight;
            for (u32 g = 0; g < kp / 32; ++g) {
                f32x4 v[2] = {};
                u32 top = 0;
#pragma unroll
                for (u32 e = 0; e < 2; ++e) {
                    if (32 * g + 8 * eight + 4 * e < pitch) v[e] = *reinterpret_cast<const f32x4 *>(row + 32 * g + 4 * e);
#pragma unroll
                    for (u32 h = 0; h < 4; ++h) {
                        const u32 b = __float_as_uint(v[e][h]) & 0x7fffffffu;
                        top = top > b ? top : b;
                    }
                }
                u32 other = wave_dpp<0xB1, 0xf>(0u, top);           // lanes 1 0 3 2
                top = top > other ? top : other;
                other = wave_dpp<0x4E, 0xf>(0u, top);               // lanes 2 3 0 1
                top = top > other ? top : other;
                const u32 scale = scale_of_max(top);
                const float inv = inverse_step(scale);
                if (m >= left) continue;
                typedef __attribute__((ext_vector_type(2))) u32 u32x2;
                *reinterpret_cast<u32x2 *>(codes + 32 * g) =
                    u32x2{pack_codes(code_of(v[0][0], inv), code_of(v[0][1], inv), code_of(v[0][2], inv), code_of(v[0][3], inv)),
                          pack_codes(code_of(v[1][0], inv), code_of(v[1][1], inv), code_of(v[1][2], inv), code_of(v[1][3], inv))};
                if (eight == 0) scales[g] = (uint8_t)scale;
            }
        }
        f32x4 acc[CT];
#pragma unroll
        for (u32 c = 0; c < CT; ++c) acc[c] = inside ? *reinterpret_cast<const f32x4 *>(lb + 16 * c + 4 * q) : f32x4{};
        if (inside) {
            for (u32 s = 0; s < steps; ++s) {
                const float v = lx[j * pitch + 4 * s + q];
#pragma unroll
                for (u32 c = 0; c < CT; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(lw[(s * CT + c) * kWave + lane], v, acc[c], 0, 0, 0);
            }
        }
        // The next tile takes this one's place before the results leave: what is waited for there is then this tile's loads and
        // not its stores.
        wave_meets();
        tile_of_x.put(lx);
        request(tile + 8);
        char *out = reinterpret_cast<char *>(static_cast<float *>(r.out) + (u64)(row0 + base) * r.ldo);
        const char *gate = static_cast<const char *>(r.gate) + (u64)(row0 + base) * r.ldgate * (GATE == 1 ? sizeof(float) : 1);
        const uint8_t *gate_scale = r.gate_scale + (GATE == 2 ? (u64)(row0 + base) * (r.ldgate / 32) : 0);
        if (j < left) {
            const u32 row = j, to = row * (u32)r.ldo;
#pragma unroll
            for (u32 c = 0; c < CT; ++c) {
                const u32 col = 16 * c + 4 * q;
                if (col >= r.cols) continue;
                f32x4 y = acc[c];
                if (r.relu) {
#pragma unroll
                    for (u32 v = 0; v < 4; ++v) y[v] = y[v] < 0.0f ? 0.0f : y[v];          // NaN stays
                }
                if (GATE == 1 && inside) {
                    const f32x4 g = load4_of(reinterpret_cast<const float *>(gate) + row * (u32)r.ldgate, col, r.cols);
#pragma unroll
                    for (u32 v = 0; v < 4; ++v) y[v] = g[v] <= 0.0f ? 0.0f : y[v];
                }
                if (GATE == 2 && inside) {
                    const u32 at = row * (u32)r.ldgate + col, g = *reinterpret_cast<const u32 *>(gate + at);
                    const bool open = gate_scale[at / 32] == 255;
#pragma unroll
                    for (u32 v = 0; v < 4; ++v) y[v] = open || (int)(signed char)(g >> (8 * v)) > 0 ? y[v] : 0.0f;
                }
                float *p = reinterpret_cast<float *>(out + (to + col) * (u32)sizeof(float));
                if (col + 4 <= r.cols) {
                    store4(p, y);
                } else {
#pragma unroll
                    for (u32 v = 0; v < 3; ++v)
                        if (col + v < r.cols) p[v] = y[v];
                }
            }
        }
    }
}

// weights, bias, four wavefronts' tiles
u32 narrow_lds_floats(u32 sums, u32 ct) { return (sums + 3) / 4 * ct * kWave + ct * 16 + 4 * kTileRows * pitch_of(sums); }

template <u32 CT, u32 PIECES>
hipError_t narrow_go(RowsArgs r, hipStream_t stream)
{
    const u32 lds = narrow_lds_floats(r.sums, CT) * 4;
    const u32 gate = !r.gate ? 0 : r.gate_scale ? 2 : 1;
    auto kernel = r.keep_codes ? narrow_rows_kernel<CT, PIECES, true, 0> : gate == 0 ? narrow_rows_kernel<CT, PIECES, false, 0>
                  : gate == 1 ? narrow_rows_kernel<CT, PIECES, false, 1> : narrow_rows_kernel<CT, PIECES, false, 2>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((u32)max_runs(r.rows, r.blocks, r.per)), dim3(256), lds, stream, r);
    return hipGetLastError();
}
template <u32 CT>
hipError_t narrow_sums(const RowsArgs &r, hipStream_t stream)
{
    if (r.sums <= 36) return narrow_go<CT, turns_of(9)>(r, stream);
    if (r.sums <= 64) return narrow_go<CT, turns_of(16)>(r, stream);
    return narrow_go<CT, turns_of(32)>(r, stream);
}
// tiles of 16 columns, as the kernels are built for them
u32 column_tiles(u32 cols)
{
    const u32 ct = (cols + 15) / 16;
    return ct == 7 ? 8 : ct;
}
hipError_t narrow_as(const RowsArgs &r, hipStream_t stream)
{
    switch (column_tiles(r.cols)) {
    case 1: return narrow_sums<1>(r, stream);
    case 2: return narrow_sums<2>(r, stream);
    case 3: return narrow_sums<3>(r, stream);
    case 4: return narrow_sums<4>(r, stream);
    case 5: return narrow_sums<5>(r, stream);
    case 6: return narrow_sums<6>(r, stream);
    default: return narrow_sums<8>(r, stream);
    }
}

}  // namespace

// At most half of a compute unit's LDS: with one workgroup there, nothing hides what its wavefronts wait for (300 000 rows, this kernel
// / the general one: 128 x 128 179 / 134 us, 104 x 108 152 / 127; with two, 96 x 96, 75 / 99).
bool narrow_rows_fit(const RowsArgs &r)
{
    if (r.cols > 128 || r.sums < 4 || r.sums > 128) return false;
    if (narrow_lds_floats(r.sums, column_tiles(r.cols)) * 4 > kLdsBytes / 2) return false;
    return r.lda <= kNarrowStride && r.ldo <= kNarrowStride && (!r.gate || r.ldgate <= kNarrowStride);
}

// Rows of a run, whole tiles for each of the four wavefronts: all runs at once, in as many workgroups a compute unit as LDS holds, four
// at most, which is what the kernels' registers leave
static u32 rows_of_run(const RowsArgs &r)
{
    const u32 lds = (narrow_lds_floats(r.sums, column_tiles(r.cols)) * 4 + kLdsPiece - 1) / kLdsPiece * kLdsPiece, held = kLdsBytes / lds;
    const u32 most = 256 * (held < 4 ? held : 4), slots = most - (r.blocks < most / 2 ? r.blocks : most / 2);
    return (u32)(((u64)r.rows + slots * 64 - 1) / (slots * 64)) * 64;
}

u64 narrow_rows_threads(const RowsArgs &r) { return max_runs(r.rows, r.blocks, rows_of_run(r)) * 256; }

hipError_t launch_narrow_rows(RowsArgs r, bool across, hipStream_t stream)
{
    r.across = across;
    r.per = rows_of_run(r);
    return narrow_as(r, stream);
}

}  // namespace lmk
