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
#include "grouped_narrow_bwd.h"

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

// CN, CK: 16 outputs and 16 inputs each
template <u32 CN, u32 CK, bool CODES>
__global__ __launch_bounds__(256, resident(CN, CK)) void narrow_backward_kernel(const BackwardArgs r)
{
    extern __shared__ __align__(16) float narrow_lds[];
    const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    if (blockIdx.x >= r.runs) {
        fill_outside(r.offsets, r.blocks, r.rows, blockIdx.x - r.runs, r.dx, r.lddx, r.k);
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
    NarrowSums<CN, CK> sums = {};
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
        sums.add(ly, pn, lx, pk, j, q);
        f32x4 acc[CK] = {};
        if (r.dx) {
            narrow_dx(acc, ly, pn, lw, steps, lane, j, q);
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
        if (r.dx && j < left) store_row(r.dx + (u64)(row0 + base) * r.lddx + j * (u32)r.lddx, acc, r.k, q);
    }
    const u32 size = r.n * r.k;
    float *set = r.part + (u64)run.partial() * (size + r.n);
    sums.join(narrow_lds, wave, j, q, r.n, r.k, r.in_major != 0, r.dw ? run.whole ? r.dw + (u64)run.block * size : set : nullptr,
              r.db ? run.whole ? r.db + (u64)run.block * r.n : set + size : nullptr);
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
