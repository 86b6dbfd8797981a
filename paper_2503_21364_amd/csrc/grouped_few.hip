// Grouped layers over few rows: a handful of anchors, most blocks without any.  Reading the weights is all of it, so a workgroup
// takes 16 rows and NT columns of the output and its eight wavefronts share out the sum indices: every wavefront streams its part
// of the weights straight into registers, whole lines a row, many loads in flight, and the parts meet in LDS.  One row and 8 blocks
// of 1024 x 1024 in bfloat16: 4.1 us, a chain of latencies; 1024 rows and 64 blocks of 1024 x 2048: 59 us (4.6 TB/s).
//
// Products by v_mfma_f32_16x16x4_f32 (products and sums in 32 bits, bfloat16 widened: 9 TB/s of bfloat16 weights
// at its rate, more than memory gives).  A step takes sum indices {q V + e : lane group q} for e = 0 .. V-1, any
// order being as good, so that a lane's x and, where the sum index is contiguous, its weights are V consecutive
// values; where the columns are contiguous a lane has NT / 16 consecutive ones, which are as many results' row.
#include "grouped_kernels.h"

namespace lmk {

namespace {

constexpr u32 kRows = 16;

// GATE: 0 none, 1 values, 2 codes
template <class T, u32 NT, bool ACROSS, Ends ENDS, u32 GATE>
__global__ __launch_bounds__(512, ENDS == Ends::whole ? 6 : 4) void few_rows_kernel(const RowsArgs r)
{
    constexpr u32 kWaves = 8, kC = NT / 16, V = ACROSS ? 4 : 16 / sizeof(T), kAhead = NT == 64 ? 2 : 4;
    __shared__ float part[kWaves][kRows][NT + 1];
    const u32 row_tile = blockIdx.x / r.col_tiles, col0 = (blockIdx.x - row_tile * r.col_tiles) * NT;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kRows, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kRows;
    const u32 height = run.end - row0 < kRows ? run.end - row0 : kRows;
    const u32 width = r.cols - col0 < NT ? r.cols - col0 : NT;
    const u32 lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), j = lane & 15, q = lane >> 4;
    const bool inside = run.block != ~0u;
    if (inside) {
        f32x4 acc[kC] = {};
        const T *x = static_cast<const T *>(r.a) + (u64)(row0 + (j < height ? j : 0)) * r.lda;
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        // this wavefront's sum indices, in steps of 4 V; a row that is not there adds nothing but garbage to results that are not written
        constexpr u32 step = 4 * V;
        const u32 all = (r.sums + step - 1) / step, per = (all + kWaves - 1) / kWaves;
        const u32 first = wave * per, last = first + per < all ? first + per : all;
        Run<T, V> fx[kAhead];
        Run<T, V> along[kAhead][kC];                    // weights: V sum indices of a column,
        Run<T, kC> across[kAhead][V];                   // or kC columns of a sum index: the last ones of the row where fewer are left
        const u32 own = kC * j < width ? kC * j : 0u, left = r.cols - col0;
        const int col = ENDS == Ends::any && own + kC > left ? (int)left - (int)kC : (int)own;
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V;
                const bool on = t0 + a < last;
                if (ENDS == Ends::any && !on) break;            // the same in all lanes
                const u32 sums = on ? r.sums : 0u;
                fx[a] = load_run<T, V, ENDS>(x, s, sums);
                if constexpr (ACROSS && ENDS == Ends::any) {
#pragma unroll
                    for (u32 e = 0; e < V; ++e) across[a][e] = load_any<Run<T, kC>>(w + (u64)(s + e < sums ? s + e : sums - 1) * r.ldw + col0 + col);
                } else if constexpr (ACROSS) {
#pragma unroll
                    for (u32 e = 0; e < V; ++e) across[a][e] = load_run<T, kC, ENDS>(w + (u64)(s + e) * r.ldw + col0, kC * j, s + e < sums ? width : 0u);
                } else {
#pragma unroll
                    for (u32 c = 0; c < kC; ++c) {
                        const u32 n = 16 * c + j;
                        along[a][c] = load_run<T, V, ENDS>(w + (u64)(col0 + (n < width ? n : 0)) * r.ldw, s, sums);
                    }
                }
            }
            if (ENDS == Ends::any && (t0 + kAhead > last || (t0 + kAhead) * step > r.sums)) {
#pragma unroll
                for (u32 a = 0; a < kAhead; ++a) {
                    const u32 s = t0 + a < last ? (t0 + a) * step + q * V : r.sums;
                    in_place<T, V>(fx[a], s, r.sums);
#pragma unroll
                    for (u32 c = 0; c < kC; ++c)
                        if constexpr (!ACROSS) in_place<T, V>(along[a][c], s, r.sums);
#pragma unroll
                    for (u32 e = 0; e < V; ++e)
                        if (ACROSS && s + e >= r.sums) across[a][e] = Run<T, kC>{};
                }
            }
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a)
#pragma unroll
                for (u32 e = 0; e < V; ++e)
#pragma unroll
                    for (u32 c = 0; c < kC; ++c)
                        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(to_f32(fx[a][e]), to_f32(ACROSS ? across[a][e][c] : along[a][c][e]), acc[c], 0, 0, 0);
        }
        // result c: rows 4 q .. 4 q + 3, column j of it
#pragma unroll
        for (u32 c = 0; c < kC; ++c)
#pragma unroll
            for (u32 v = 0; v < 4; ++v) {
                // columns in front of the tile are another one's
                const int at = !ACROSS ? (int)(16 * c + j) : ENDS == Ends::any ? col + (int)c : (int)(kC * j + c);
                if (!ACROSS || ENDS != Ends::any || (at >= 0 && kC * j < width)) part[wave][4 * q + v][at] = acc[c][v];
            }
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < kRows * NT; i += 512) {
        const u32 row = i / NT, c = i % NT;
        if (row >= height || c >= width) continue;
        float y = 0.0f;
        if (inside) {
#pragma unroll
            for (u32 p = 0; p < kWaves; ++p) y += part[p][row][c];
            if (r.bias) y += r.bias[(u64)run.block * r.cols + col0 + c];
            if (r.relu) y = y < 0.0f ? 0.0f : y;              // NaN stays
            const u64 at = (u64)(row0 + row) * r.ldgate + col0 + c;
            if (GATE == 1) y = to_f32(static_cast<const T *>(r.gate)[at]) <= 0.0f ? 0.0f : y;
            if (GATE == 2) y = (static_cast<const signed char *>(r.gate)[at] > 0 || r.gate_scale[at / 32] == 255) ? y : 0.0f;
        }
        static_cast<T *>(r.out)[(u64)(row0 + row) * r.ldo + col0 + c] = (T)y;
    }
}

template <class T, u32 NT, bool ACROSS, Ends ENDS, u32 GATE>
hipError_t few_go(RowsArgs r, hipStream_t stream)
{
    r.col_tiles = (r.cols + NT - 1) / NT;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kRows) * r.col_tiles);
    hipLaunchKernelGGL((few_rows_kernel<T, NT, ACROSS, ENDS, GATE>), dim3(r.tiles), dim3(512), 0, stream, r);
    return hipGetLastError();
}
// Columns of a workgroup.  64 make whole lines where columns are contiguous (8 blocks of 1024 x 1024 in bfloat16, 128 rows, 64 / 16
// columns: 10.5 / 14.3 us; one row: 8.9 / 5.3), and read x once for four results where they are not (one block of 2048 x 2048
// in float32, 128 rows: 24 / 31 us); 16 where that leaves compute units without work (8 blocks of 1024 x 1024, 128 rows: 10.3 / 7.0)
u32 few_columns(const RowsArgs &r, bool across)
{
    return max_runs(r.rows, r.blocks, kRows) * ((r.cols + 63) / 64) >= (across ? 64 : 320) ? 64 : 16;
}
template <class T, bool ACROSS, u32 GATE>
hipError_t few_width(const RowsArgs &r, hipStream_t stream)
{
    constexpr u32 v = ACROSS ? 4 : 16 / sizeof(T);          // a run of x, and of the weights
    const bool wide = few_columns(r, ACROSS) == 64;
    const Ends sums = ends_of(r.sums, v), cols = ACROSS && wide ? ends_of(r.cols, 4) : Ends::whole;
    // value by value where a row is a few vectors of four, and so many columns share a line (408 rows of 76 blocks -> 1715 in float32, 15 inputs: 10.8 us,
    // by vectors 12.9; 47: 15.1 and 15.2; 61: 16.6 and 15.6; 200 rows of 20 in bfloat16, eight to a vector, 15 inputs: 8.5 and 7.8)
    const bool single = sizeof(T) == 4 && !ACROSS && sums == Ends::any && r.sums < 48;
    if (single || sums == Ends::early || cols == Ends::early)
        return wide ? few_go<T, 64, ACROSS, Ends::early, GATE>(r, stream) : few_go<T, 16, ACROSS, Ends::early, GATE>(r, stream);
    if (sums == Ends::any || cols == Ends::any)
        return wide ? few_go<T, 64, ACROSS, Ends::any, GATE>(r, stream) : few_go<T, 16, ACROSS, Ends::any, GATE>(r, stream);
    return wide ? few_go<T, 64, ACROSS, Ends::whole, GATE>(r, stream) : few_go<T, 16, ACROSS, Ends::whole, GATE>(r, stream);
}
template <class T>
hipError_t few_as(const RowsArgs &r, bool across, hipStream_t stream)
{
    const u32 gate = !r.gate ? 0 : r.gate_scale ? 2 : 1;
    if (across) return gate == 0 ? few_width<T, true, 0>(r, stream) : gate == 1 ? few_width<T, true, 1>(r, stream) : few_width<T, true, 2>(r, stream);
    return gate == 0 ? few_width<T, false, 0>(r, stream) : gate == 1 ? few_width<T, false, 1>(r, stream) : few_width<T, false, 2>(r, stream);
}

}  // namespace

// Where the other kernels' tiles would be mostly empty, or too few.  This kernel / the bfloat16 one, forward: one block of 2048 x 2048,
// 128 rows 17 / 25 us, 256 rows 29 / 25; 24 blocks of 512 x 512, 256 rows 6.6 / 8.0, 512 rows 9.5 / 8.1; but 64 blocks of
// 1024 x 2048, whose tiles fill the device with a row each, 64 rows 52 / 43, 1024 rows 58 / 45.  This one / the float32 ones:
// one block of 2048 x 2048, 512 rows 88 / 108, 1024 rows 169 / 144; 8 blocks of 1024 x 1024, 1024 rows 48 / 58, 2048 rows
// 90 / 75; 24 blocks of 96 x 35, 4096 rows 6.4 / 7.7, 8192 rows 9.6 / 7.9.
bool few_rows_fit(const RowsArgs &r, bool wide)
{
    if (!wide) return r.rows <= 4096 && r.rows / 64 <= r.blocks + 8;
    const u64 row_tiles = r.rows < r.blocks ? r.rows : r.blocks;
    return (r.rows <= 128 || r.rows / 16 <= r.blocks) && row_tiles * ((r.cols + 127) / 128) < 512;
}

u64 few_rows_threads(const RowsArgs &r, bool across)
{
    const u32 nt = few_columns(r, across);
    return max_runs(r.rows, r.blocks, kRows) * ((r.cols + nt - 1) / nt) * 512;
}

hipError_t launch_few_rows(const RowsArgs &r, u32 dtype, bool across, hipStream_t stream)
{
    return dtype == LMK_GS_F32 ? few_as<float>(r, across, stream) : few_as<__bf16>(r, across, stream);
}

}  // namespace lmk
