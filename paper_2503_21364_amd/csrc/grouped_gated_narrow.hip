// Gated layers whose weights are small, in float32 (the decoder's sizes): memory is all of it, so a row is read once and its results leave
// once.  As in grouped_narrow.hip a workgroup keeps its block's matrices in LDS and its four wavefronts walk through a run of the block's
// rows in tiles of 16, each by itself; a lane has both projections of the same four outputs of a row.
//
// All gradients are one kernel, too: both projections of a tile, their gradients from there into LDS, side by side, in the place that
// grouped_narrow_bwd.hip has a tile of dy in, and dx, dw and db as there.  They never go to memory.
//
// 300 000 rows in 24 blocks: 35 -> 32 32 us (80 MB, 2.5 TB/s; the general kernel 60), 96 -> 32 61 (91).  All gradients 81 (147) for 35 -> 32, 188
// (253) for 64 -> 48: half of the float32 instructions' rate, counting their padding to tiles of 16; a wavefront's tile is a chain through LDS, and
// the sums' registers leave two or three wavefronts a SIMD to fill its waits.
#include "grouped_gated.h"
#include "grouped_narrow_bwd.h"

namespace lmk {

namespace {

// Both projections of a tile of x: `cg` tiles of 16 outputs.  Weights in LDS: the gate's, then the others'; bias: 16 CG each
template <u32 CG>
__device__ __forceinline__ void project(f32x4 (&a)[CG], f32x4 (&u)[CG], const float *lw, const float *lb, const float *lx, u32 pk, u32 steps,
                                        u32 lane, u32 j, u32 q)
{
#pragma unroll
    for (u32 c = 0; c < CG; ++c) {
        a[c] = *reinterpret_cast<const f32x4 *>(lb + 16 * c + 4 * q);
        u[c] = *reinterpret_cast<const f32x4 *>(lb + 16 * (CG + c) + 4 * q);
    }
    const float *lu = lw + steps * CG * kWave;
    for (u32 s = 0; s < steps; ++s) {
        const float v = lx[j * pk + 4 * s + q];
#pragma unroll
        for (u32 c = 0; c < CG; ++c) {
            a[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(lw[(s * CG + c) * kWave + lane], v, a[c], 0, 0, 0);
            u[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(lu[(s * CG + c) * kWave + lane], v, u[c], 0, 0, 0);
        }
    }
}
// a block's weights and bias for it
template <u32 CG> __device__ __forceinline__ void stage_projections(float *lw, float *lb, const GatedArgs &r, u32 block, u32 steps)
{
    const float *w = static_cast<const float *>(r.w) + (u64)block * r.w_block;
    stage_weights<float, CG>(lw, w, r.ldw, r.in_major, r.k, r.n);
    stage_weights<float, CG>(lw + steps * CG * kWave, w + (r.in_major ? (u64)r.n : (u64)r.n * r.ldw), r.ldw, r.in_major, r.k, r.n);
    for (u32 i = threadIdx.x; i < 2 * CG * 16; i += 256) {
        const u32 h = i / (CG * 16), c = i % (CG * 16);
        lb[i] = r.bias && c < r.n ? r.bias[(u64)block * 2 * r.n + h * r.n + c] : 0.0f;
    }
}
__host__ __device__ constexpr u32 projection_floats(u32 k, u32 cg) { return (k + 3) / 4 * 2 * cg * kWave + 2 * cg * 16; }

// PIECES: turns in which a wavefront brings a tile of x
template <u32 CG, u32 PIECES>
__global__ __launch_bounds__(256, 3) void gated_narrow_kernel(const GatedArgs r, u32 per)
{
    extern __shared__ __align__(16) float narrow_lds[];
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, per, blockIdx.x);
    if (!run.found) return;
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), j = lane & 15, q = lane >> 4;
    const u32 row0 = run.begin + run.local * per;
    const u32 height = run.end - row0 < per ? run.end - row0 : per;
    const bool inside = run.block != ~0u;
    const u32 steps = (r.k + 3) / 4, pk = pitch_of(r.k);
    float *lw = narrow_lds, *lb = lw + steps * 2 * CG * kWave, *lx = lb + 2 * CG * 16 + wave * kTileRows * pk;
    if (inside) stage_projections<CG>(lw, lb, r, run.block, steps);
    __syncthreads();
    const u32 tiles = (height + kTileRows - 1) / kTileRows;
    const char *x = reinterpret_cast<const char *>(static_cast<const float *>(r.x) + (u64)row0 * r.ldx);
    Pieces<float, PIECES> tile_of_x;
    tile_of_x.init(r.ldx, r.k, lane);
    clear_gaps(lx, r.k, lane);
    auto request = [&](u32 tile) {
        tile_of_x.request(x + (u64)tile * kTileRows * r.ldx * sizeof(float), inside && tile < tiles ? height - tile * kTileRows : 0u);
    };
    request(wave);
    tile_of_x.put(lx);
    request(wave + 4);
    for (u32 tile = wave; tile < tiles; tile += 4) {
        const u32 base = tile * kTileRows, left = height - base;
        wave_meets();
        f32x4 a[CG] = {}, u[CG] = {};
        if (inside) project<CG>(a, u, lw, lb, lx, pk, steps, lane, j, q);
        // the next tile takes this one's place before the results leave
        wave_meets();
        tile_of_x.put(lx);
        request(tile + 8);
#pragma unroll
        for (u32 c = 0; c < CG; ++c)
#pragma unroll
            for (u32 v = 0; v < 4; ++v) a[c][v] = inside ? gated(r.act, a[c][v], u[c][v]) : 0.0f;
        if (j < left) store_row(static_cast<float *>(r.out) + (u64)(row0 + base) * r.ldo + j * (u32)r.ldo, a, r.n, q);
    }
}

// Workgroups of a compute unit by LDS; the registers leave three up to twelve tiles of sums, two up to 24
constexpr u32 backward_floats(u32 n, u32 k, u32 cg, u32 cn, u32 ck)
{
    const u32 before = whole_steps(2 * n) * ck * kWave + projection_floats(k, cg) + 4 * kTileRows * (pitch_of(2 * n) + pitch_of(k));
    const u32 sums = 4 * sums_floats(cn, ck);
    return before > sums ? before : sums;
}
constexpr u32 gated_resident(u32 cg, u32 ck)
{
    const u32 lds = kLdsBytes / ((backward_floats(16 * cg, 16 * ck, cg, 2 * cg, ck) * 4 + kLdsPiece - 1) / kLdsPiece * kLdsPiece);
    const u32 registers = 2 * cg * ck <= 12 ? 3 : 2;
    return lds < 1 ? 1 : registers < lds ? registers : lds;
}

struct GatedNarrowGrads {
    float *dx;
    u64 lddx;
    float *dw, *db, *part;      // any of the first three may be NULL
    u32 runs, per;
};

// CG: 16 outputs of each projection, CK: 16 inputs
template <u32 CG, u32 CK>
__global__ __launch_bounds__(256, gated_resident(CG, CK)) void gated_narrow_backward_kernel(const GatedArgs r, const GatedNarrowGrads g)
{
    extern __shared__ __align__(16) float narrow_lds[];
    constexpr u32 CN = 2 * CG;
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    if (blockIdx.x >= g.runs) {
        fill_outside(r.offsets, r.blocks, r.rows, blockIdx.x - g.runs, g.dx, g.lddx, r.k);
        return;
    }
    const u32 n2 = 2 * r.n, pn = pitch_of(n2), pk = pitch_of(r.k), out_steps = (n2 + 3) / 4, steps = (r.k + 3) / 4;
    float *lw = narrow_lds, *lp = lw + whole_steps(n2) * CK * kWave, *lb = lp + steps * 2 * CG * kWave;
    float *ly = lb + 2 * CG * 16 + wave * kTileRows * (pn + pk), *lx = ly + kTileRows * pn;
    BlockRun run;
    if (!run.find(r.offsets, r.blocks, r.rows, g.per, blockIdx.x)) return;
    const u32 row0 = run.row, height = run.count, lane = threadIdx.x & (kWave - 1), j = lane & 15, q = lane >> 4;
    const float *w = static_cast<const float *>(r.w) + (u64)run.block * r.w_block;
    if (g.dx) {
        stage_weights<float, CK>(lw, w, r.ldw, !r.in_major, n2, r.k);
        for (u32 i = out_steps * CK * kWave + threadIdx.x; i < whole_steps(n2) * CK * kWave; i += 256) lw[i] = 0.0f;
    }
    stage_projections<CG>(lp, lb, r, run.block, steps);
    __syncthreads();

    const u32 tiles = (height + kTileRows - 1) / kTileRows;
    const char *x = reinterpret_cast<const char *>(static_cast<const float *>(r.x) + (u64)row0 * r.ldx);
    const float *dy = static_cast<const float *>(r.dy) + (u64)row0 * r.lddy;
    Pieces<float, turns_of(4 * CK)> tile_x;
    tile_x.init(r.ldx, r.k, lane);
    clear_gaps(lx, r.k, lane);
    // behind both projections' gradients, too: a weight's zero times what lies there would be NaN for a NaN
    if (lane < kTileRows)
        for (u32 c = n2; c < pn; ++c) ly[lane * pn + c] = 0.0f;
    f32x4 next[CG] = {};
    auto request = [&](u32 tile) {
        const u32 rows = tile < tiles ? height - tile * kTileRows : 0u;
        tile_x.request(x + (u64)tile * kTileRows * r.ldx * 4, rows);
        if (rows == 0) return;
        // four outputs of a row a lane, as the projections have them; a row that is not there is read as the tile's first
        const float *from = dy + ((u64)tile * kTileRows + (j < rows ? j : 0u)) * r.lddy;
#pragma unroll
        for (u32 c = 0; c < CG; ++c) next[c] = 16 * c + 4 * q < r.n ? load4_of(from, 16 * c + 4 * q, r.n) : f32x4{};
    };
    NarrowSums<CN, CK> sums = {};
    request(wave);
    tile_x.put(lx);
    f32x4 up[CG];
#pragma unroll
    for (u32 c = 0; c < CG; ++c) up[c] = next[c];
    request(wave + 4);
    for (u32 tile = wave; tile < tiles; tile += 4) {
        const u32 base = tile * kTileRows, left = height - base;
        wave_meets();
        {
            f32x4 a[CG], u[CG];
            project<CG>(a, u, lp, lb, lx, pk, steps, lane, j, q);
#pragma unroll
            for (u32 c = 0; c < CG; ++c) {
                const u32 at = 16 * c + 4 * q;
                if (at >= r.n) continue;
                f32x4 da, du;
#pragma unroll
                for (u32 v = 0; v < 4; ++v) {
                    float ga, gu;
                    gated_gradient(r.act, a[c][v], u[c][v], up[c][v], ga, gu);
                    da[v] = j < left ? ga : 0.0f;
                    du[v] = j < left ? gu : 0.0f;
                }
                float *to = ly + j * pn + at;
                if (r.n % 4 == 0) {
                    *reinterpret_cast<f32x4 *>(to) = da;
                    *reinterpret_cast<f32x4 *>(to + r.n) = du;
                } else {
#pragma unroll
                    for (u32 v = 0; v < 4; ++v)
                        if (at + v < r.n) {
                            to[v] = da[v];
                            to[r.n + v] = du[v];
                        }
                }
            }
        }
        wave_meets();
        sums.add(ly, pn, lx, pk, j, q);
        f32x4 acc[CK] = {};
        if (g.dx) narrow_dx(acc, ly, pn, lw, out_steps, lane, j, q);
        // the next tile takes this one's place before the results leave
        wave_meets();
        tile_x.put(lx);
#pragma unroll
        for (u32 c = 0; c < CG; ++c) up[c] = next[c];
        request(tile + 8);
        if (g.dx && j < left) store_row(g.dx + (u64)(row0 + base) * g.lddx + j * (u32)g.lddx, acc, r.k, q);
    }
    const u32 size = n2 * r.k;
    float *set = g.part + (u64)run.partial() * (size + n2);
    sums.join(narrow_lds, wave, j, q, n2, r.k, r.in_major, g.dw ? run.whole ? g.dw + (u64)run.block * size : set : nullptr,
              g.db ? run.whole ? g.db + (u64)run.block * n2 : set + size : nullptr);
}

// ---- launches
u32 output_tiles(u32 n) { return (n + 15) / 16; }

template <u32 CG, u32 PIECES> hipError_t narrow_go(const GatedArgs &r, u32 per, hipStream_t stream)
{
    const u32 lds = (projection_floats(r.k, CG) + 4 * kTileRows * pitch_of(r.k)) * 4;
    auto kernel = gated_narrow_kernel<CG, PIECES>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((u32)max_runs(r.rows, r.blocks, per)), dim3(256), lds, stream, r, per);
    return hipGetLastError();
}
template <u32 CG> hipError_t narrow_k(const GatedArgs &r, u32 per, hipStream_t stream)
{
    if (r.k <= 36) return narrow_go<CG, turns_of(9)>(r, per, stream);
    if (r.k <= 64) return narrow_go<CG, turns_of(16)>(r, per, stream);
    return narrow_go<CG, turns_of(32)>(r, per, stream);
}

// Rows of a run, whole tiles for each of the four wavefronts: all runs at once
u32 rows_of_run(u32 rows, u32 blocks, u32 most)
{
    const u32 slots = most - (blocks < most / 2 ? blocks : most / 2);
    const u32 per = (u32)(((u64)rows + slots * 64 - 1) / (slots * 64)) * 64;
    return per < 64 ? 64 : per;
}
u32 forward_rows(const GatedArgs &r)
{
    const u32 lds = ((projection_floats(r.k, output_tiles(r.n)) + 4 * kTileRows * pitch_of(r.k)) * 4 + kLdsPiece - 1) / kLdsPiece * kLdsPiece;
    const u32 held = kLdsBytes / lds;
    return rows_of_run(r.rows, r.blocks, 256 * (held < 3 ? held : 3));
}

template <u32 CG, u32 CK> hipError_t backward_go(const GatedArgs &r, const GatedNarrowGrads &g, hipStream_t stream)
{
    const u32 lds = backward_floats(r.n, r.k, CG, 2 * CG, CK) * 4;
    auto kernel = gated_narrow_backward_kernel<CG, CK>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(g.runs + kFillers), dim3(256), lds, stream, r, g);
    return hipGetLastError();
}
template <u32 CG> hipError_t backward_k(const GatedArgs &r, const GatedNarrowGrads &g, hipStream_t stream)
{
    switch ((r.k + 15) / 16) {
    case 1: return backward_go<CG, 1>(r, g, stream);
    case 2: return backward_go<CG, 2>(r, g, stream);
    case 3: return backward_go<CG, 3>(r, g, stream);
    default: return backward_go<CG, 4>(r, g, stream);
    }
}

}  // namespace

// At most half of a compute unit's LDS, as narrow_rows_fit
bool gated_narrow_fits(const GatedArgs &r)
{
    if (r.n > 64 || r.n < 4 || r.k < 4 || r.k > 128 || r.ldx > kNarrowStride || r.ldo > kNarrowStride) return false;
    return (projection_floats(r.k, output_tiles(r.n)) + 4 * kTileRows * pitch_of(r.k)) * 4 <= kLdsBytes / 2;
}
u64 gated_narrow_threads(const GatedArgs &r) { return max_runs(r.rows, r.blocks, forward_rows(r)) * 256; }

hipError_t launch_gated_narrow(const GatedArgs &r, hipStream_t stream)
{
    const u32 per = forward_rows(r);
    switch (output_tiles(r.n)) {
    case 1: return narrow_k<1>(r, per, stream);
    case 2: return narrow_k<2>(r, per, stream);
    case 3: return narrow_k<3>(r, per, stream);
    default: return narrow_k<4>(r, per, stream);
    }
}

bool gated_narrow_backward_fits(const GatedArgs &r, u64 lddx)
{
    return r.n >= 4 && r.n <= 48 && r.k >= 4 && r.k <= 64 && r.ldx <= kNarrowStride && r.lddy <= kNarrowStride && lddx <= kNarrowStride;
}
u32 gated_narrow_backward_rows(const GatedArgs &r)
{
    const u32 cg = output_tiles(r.n), ck = (r.k + 15) / 16;
    return rows_of_run(r.rows, r.blocks, 256 * gated_resident(cg, ck));
}
hipError_t launch_gated_narrow_backward(const GatedArgs &r, float *dx, u64 lddx, float *dw, float *db, float *part, hipStream_t stream)
{
    GatedNarrowGrads g = {dx, lddx, dw, db, part, 0, gated_narrow_backward_rows(r)};
    g.runs = r.rows / g.per + 1 + r.blocks;
    switch (output_tiles(r.n)) {
    case 1: return backward_k<1>(r, g, stream);
    case 2: return backward_k<2>(r, g, stream);
    default: return backward_k<3>(r, g, stream);
    }
}

}  // namespace lmk
