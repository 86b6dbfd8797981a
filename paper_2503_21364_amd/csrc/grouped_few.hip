// Grouped layers over few rows: a handful of anchors, most blocks without any.  Reading the weights is all of it, so a workgroup
// takes 16 rows and NT columns of the output and its eight wavefronts share out the sum indices: every wavefront streams its part
// of the weights straight into registers, whole lines a row, many loads in flight, and the parts meet in LDS.
//
// Products by v_mfma_f32_16x16x4_f32 (products and sums in 32 bits, bfloat16 widened: 9 TB/s of bfloat16 weights
// at its rate, more than memory gives).  A step takes sum indices {q V + e : lane group q} for e = 0 .. V-1, any
// order being as good, so that a lane's x and, where the sum index is contiguous, its weights are V consecutive
// values; where the columns are contiguous a lane has NT / 16 consecutive ones, which are as many results' row.
#include "grouped_kernels.h"

namespace lmk {

namespace {

constexpr u32 kRows = 16;

// V values of a row from `s` on; beyond `sums` zeros.  wide: rows start at boundaries of V values (of 16 bytes at most)
template <class T, u32 V>
__device__ __forceinline__ void load_run(float (&v)[V], const T *p, u32 s, u32 sums, bool wide)
{
    if constexpr (V % 4 == 0) {
        if (wide && s + V <= sums) {
            if constexpr (V * sizeof(T) == 16) {
                typedef __attribute__((ext_vector_type(V))) T vec;
                const vec q = *reinterpret_cast<const vec *>(p + s);
#pragma unroll
                for (u32 e = 0; e < V; ++e) v[e] = to_f32(q[e]);
            } else {
                const f32x4 q = load4(p + s);
#pragma unroll
                for (u32 e = 0; e < V; ++e) v[e] = q[e];
            }
            return;
        }
    }
#pragma unroll
    for (u32 e = 0; e < V; ++e) v[e] = s + e < sums ? to_f32(p[s + e]) : 0.0f;
}

// GATE: 0 none, 1 values, 2 codes
template <class T, u32 NT, bool ACROSS, u32 GATE>
__global__ __launch_bounds__(512) void few_rows_kernel(const RowsArgs r)
{
    constexpr u32 kWaves = 8, kC = NT / 16, V = ACROSS ? 4 : 16 / sizeof(T), kAhead = (NT == 64 ? 16 : 32) / V;
    __shared__ float part[kWaves][kRows][NT + 1];
    const u32 row_tile = blockIdx.x / r.col_tiles, col0 = (blockIdx.x - row_tile * r.col_tiles) * NT;
    const RowRun run = find_run<true>(r.offsets, r.blocks, r.rows, kRows, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kRows;
    const u32 height = run.end - row0 < kRows ? run.end - row0 : kRows;
    const u32 width = r.cols - col0 < NT ? r.cols - col0 : NT;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 15, q = lane >> 4;
    const bool inside = run.block != ~0u;
    if (inside) {
        f32x4 acc[kC] = {};
        const T *x = static_cast<const T *>(r.a) + (u64)(row0 + (j < height ? j : 0)) * r.lda;
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        // this wavefront's sum indices, in steps of 4 V; a row that is not there adds nothing but garbage to results that are not written
        constexpr u32 step = 4 * V;
        const u32 all = (r.sums + step - 1) / step, per = (all + kWaves - 1) / kWaves;
        const u32 first = wave * per, last = first + per < all ? first + per : all;
        float fx[kAhead][V], fw[kAhead][kC][V];
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V;
                const bool on = t0 + a < last;
                load_run<T, V>(fx[a], x, s, on ? r.sums : 0u, r.wide_a);
#pragma unroll
                for (u32 c = 0; c < kC; ++c) {
                    if (ACROSS) continue;
                    const u32 n = 16 * c + j;
                    load_run<T, V>(fw[a][c], w + (u64)(col0 + (n < width ? n : 0)) * r.ldw, s, on ? r.sums : 0u, r.wide_w);
                }
                if constexpr (ACROSS) {
#pragma unroll
                    for (u32 e = 0; e < V; ++e) {
                        float v[kC];
                        load_run<T, kC>(v, w + (u64)(s + e) * r.ldw + col0, kC * j, on && s + e < r.sums ? width : 0u, r.wide_w);
#pragma unroll
                        for (u32 c = 0; c < kC; ++c) fw[a][c][e] = v[c];
                    }
                }
            }
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a)
#pragma unroll
                for (u32 e = 0; e < V; ++e)
#pragma unroll
                    for (u32 c = 0; c < kC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(fx[a][e], fw[a][c][e], acc[c], 0, 0, 0);
        }
        // result c: rows 4 q .. 4 q + 3, column j of it
#pragma unroll
        for (u32 c = 0; c < kC; ++c)
#pragma unroll
            for (u32 v = 0; v < 4; ++v) part[wave][4 * q + v][ACROSS ? kC * j + c : 16 * c + j] = acc[c][v];
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

template <class T, u32 NT, bool ACROSS, u32 GATE>
hipError_t few_go(RowsArgs r, hipStream_t stream)
{
    r.col_tiles = (r.cols + NT - 1) / NT;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kRows, true) * r.col_tiles);
    hipLaunchKernelGGL((few_rows_kernel<T, NT, ACROSS, GATE>), dim3(r.tiles), dim3(512), 0, stream, r);
    return hipGetLastError();
}
template <class T, bool ACROSS, u32 GATE>
hipError_t few_width(const RowsArgs &r, hipStream_t stream)
{
    // 64 columns make whole lines where columns are contiguous and read x once for four results; 16 where that leaves
    // compute units without work
    if (max_runs(r.rows, r.blocks, kRows, true) * ((r.cols + 63) / 64) >= 256) return few_go<T, 64, ACROSS, GATE>(r, stream);
    return few_go<T, 16, ACROSS, GATE>(r, stream);
}
template <class T>
hipError_t few_as(RowsArgs r, bool across, hipStream_t stream)
{
    const u32 v = across ? 4 : 16 / sizeof(T);
    const auto wide = [v](const void *p, u64 ld) { return ld % v == 0 && reinterpret_cast<uintptr_t>(p) % (v * sizeof(T)) == 0; };
    r.wide_a = wide(r.a, r.lda);
    r.wide_w = wide(r.w, r.ldw) && r.w_block % v == 0;
    const u32 gate = !r.gate ? 0 : r.gate_scale ? 2 : 1;
    if (across) return gate == 0 ? few_width<T, true, 0>(r, stream) : gate == 1 ? few_width<T, true, 1>(r, stream) : few_width<T, true, 2>(r, stream);
    return gate == 0 ? few_width<T, false, 0>(r, stream) : gate == 1 ? few_width<T, false, 1>(r, stream) : few_width<T, false, 2>(r, stream);
}

}  // namespace

bool few_rows_fit(const RowsArgs &r) { return r.rows <= 256; }

hipError_t launch_few_rows(const RowsArgs &r, u32 dtype, bool across, hipStream_t stream)
{
    return dtype == LMK_GS_F32 ? few_as<float>(r, across, stream) : few_as<__bf16>(r, across, stream);
}

}  // namespace lmk
