// Gated layers over few rows: as in grouped_few.hip a workgroup takes 16 rows and NT outputs, its eight wavefronts share out the sum
// indices and stream their part of both projections' weights straight into registers; the parts meet in LDS, where the activation and
// the product, or their gradients, are taken.
#include "grouped_gated.h"

namespace lmk {

namespace {

constexpr u32 kRows = kGatedFewRows;

// BACKWARD: the gradients of both projections instead of y
template <class T, u32 NT, bool ACROSS, bool WHOLE, bool BACKWARD>
__global__ __launch_bounds__(512, 4) void gated_few_kernel(const GatedArgs r)
{
    constexpr u32 kWaves = 8, kC = NT / 16, V = ACROSS ? 4 : 16 / sizeof(T), kAhead = NT == 32 ? 2 : 4;
    __shared__ float part[kWaves][kRows][2 * NT + 1];
    const u32 row_tile = blockIdx.x / r.col_tiles, col0 = (blockIdx.x - row_tile * r.col_tiles) * NT;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kRows, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kRows;
    const u32 height = run.end - row0 < kRows ? run.end - row0 : kRows;
    const u32 width = r.n - col0 < NT ? r.n - col0 : NT;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 15, q = lane >> 4;
    const bool inside = run.block != ~0u;
    if (inside) {
        f32x4 acc[2][kC] = {};
        const T *x = static_cast<const T *>(r.x) + (u64)(row0 + (j < height ? j : 0)) * r.ldx;
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        // this wavefront's sum indices, in steps of 4 V; a row that is not there adds nothing but garbage to results that are not written
        constexpr u32 step = 4 * V;
        const u32 all = (r.k + step - 1) / step, per = (all + kWaves - 1) / kWaves;
        const u32 first = wave * per, last = first + per < all ? first + per : all;
        Run<T, V> fx[kAhead];
        Run<T, V> along[kAhead][2][kC];                 // weights: V sum indices of a column,
        Run<T, kC> across[kAhead][2][V];                // or kC columns of a sum index
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V;
                const bool on = t0 + a < last;
                fx[a] = load_run<T, V, WHOLE>(x, s, on ? r.k : 0u);
#pragma unroll
                for (u32 h = 0; h < 2; ++h) {
                    if constexpr (ACROSS) {
#pragma unroll
                        for (u32 e = 0; e < V; ++e)
                            across[a][h][e] = load_run<T, kC, WHOLE>(w + (u64)(s + e) * r.ldw + h * r.n + col0, kC * j, on && s + e < r.k ? width : 0u);
                    } else {
#pragma unroll
                        for (u32 c = 0; c < kC; ++c) {
                            const u32 n = 16 * c + j;
                            along[a][h][c] = load_run<T, V, WHOLE>(w + (u64)(h * r.n + col0 + (n < width ? n : 0)) * r.ldw, s, on ? r.k : 0u);
                        }
                    }
                }
            }
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a)
#pragma unroll
                for (u32 e = 0; e < V; ++e)
#pragma unroll
                    for (u32 h = 0; h < 2; ++h)
#pragma unroll
                        for (u32 c = 0; c < kC; ++c)
                            acc[h][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(to_f32(fx[a][e]), to_f32(ACROSS ? across[a][h][e][c] : along[a][h][c][e]),
                                                                             acc[h][c], 0, 0, 0);
        }
        // result c: rows 4 q .. 4 q + 3, column j of it
#pragma unroll
        for (u32 h = 0; h < 2; ++h)
#pragma unroll
            for (u32 c = 0; c < kC; ++c)
#pragma unroll
                for (u32 v = 0; v < 4; ++v) part[wave][4 * q + v][h * NT + (ACROSS ? kC * j + c : 16 * c + j)] = acc[h][c][v];
    }
    __syncthreads();
    const u32 row = threadIdx.x / NT, c = threadIdx.x % NT;
    static_assert(kRows * NT <= 512, "a result a thread");
    const bool there = row < height && c < width;
    float da = 0.0f, du = 0.0f;
    if (there) {
        float v[2] = {0.0f, 0.0f};
        if (inside) {
#pragma unroll
            for (u32 h = 0; h < 2; ++h) {
#pragma unroll
                for (u32 p = 0; p < kWaves; ++p) v[h] += part[p][row][h * NT + c];
                if (r.bias) v[h] += r.bias[(u64)run.block * 2 * r.n + h * r.n + col0 + c];
            }
        }
        T *out = static_cast<T *>(r.out) + (u64)(row0 + row) * r.ldo + col0 + c;
        if constexpr (!BACKWARD) {
            out[0] = (T)(inside ? gated(r.act, v[0], v[1]) : 0.0f);
        } else {
            if (inside) gated_gradient(r.act, v[0], v[1], to_f32(static_cast<const T *>(r.dy)[(u64)(row0 + row) * r.lddy + col0 + c]), da, du);
            out[0] = (T)da;
            out[r.n] = (T)du;
        }
    }
    if constexpr (BACKWARD) {
        if (!r.part || !inside) return;                 // the whole workgroup
        __syncthreads();
        if (row < kRows) {
            part[0][row][c] = da;
            part[0][row][NT + c] = du;
        }
        __syncthreads();
        if (threadIdx.x >= 2 * NT || threadIdx.x % NT >= width) return;
        float s = 0.0f;
#pragma unroll
        for (u32 i = 0; i < kRows; ++i) s += part[0][i][threadIdx.x];
        set_of(r, run, kRows)[threadIdx.x / NT * r.n + col0 + threadIdx.x % NT] = s;
    }
}

template <class T, u32 NT, bool ACROSS, bool WHOLE>
hipError_t few_go(GatedArgs r, hipStream_t stream)
{
    r.col_tiles = (r.n + NT - 1) / NT;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kRows) * r.col_tiles);
    if (r.dy) hipLaunchKernelGGL((gated_few_kernel<T, NT, ACROSS, WHOLE, true>), dim3(r.tiles), dim3(512), 0, stream, r);
    else hipLaunchKernelGGL((gated_few_kernel<T, NT, ACROSS, WHOLE, false>), dim3(r.tiles), dim3(512), 0, stream, r);
    return hipGetLastError();
}
// Outputs of a workgroup: 32 where that fills the compute units, 16 where not
u32 few_columns(const GatedArgs &r)
{
    return max_runs(r.rows, r.blocks, kRows) * ((r.n + 31) / 32) >= 320 ? 32 : 16;
}
template <class T, bool ACROSS>
hipError_t few_width(const GatedArgs &r, hipStream_t stream)
{
    constexpr u32 v = ACROSS ? 4 : 16 / sizeof(T);          // a run of x, and of the weights
    const bool whole = r.k % v == 0 && (!ACROSS || r.n % v == 0);
    if (few_columns(r) == 32) return whole ? few_go<T, 32, ACROSS, true>(r, stream) : few_go<T, 32, ACROSS, false>(r, stream);
    return whole ? few_go<T, 16, ACROSS, true>(r, stream) : few_go<T, 16, ACROSS, false>(r, stream);
}

}  // namespace

// as few_rows_fit
bool gated_few_fit(const GatedArgs &r, bool wide)
{
    if (!wide) return r.rows <= 4096 && r.rows / 64 <= r.blocks + 8;
    const u64 row_tiles = r.rows < r.blocks ? r.rows : r.blocks;
    return (r.rows <= 128 || r.rows / 16 <= r.blocks) && row_tiles * ((r.n + 63) / 64) < 512;
}

u64 gated_few_threads(const GatedArgs &r)
{
    const u32 nt = few_columns(r);
    return max_runs(r.rows, r.blocks, kRows) * ((r.n + nt - 1) / nt) * 512;
}

hipError_t launch_gated_few(const GatedArgs &r, u32 dtype, hipStream_t stream)
{
    if (dtype == LMK_GS_F32) return r.in_major ? few_width<float, true>(r, stream) : few_width<float, false>(r, stream);
    return r.in_major ? few_width<__bf16, true>(r, stream) : few_width<__bf16, false>(r, stream);
}

}  // namespace lmk
