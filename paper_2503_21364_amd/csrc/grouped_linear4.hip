// Layers whose weights belong to blocks of rows, both operands in 4 bits (lmk_gs_grouped_linear4): y = act(x w_g^T + b_g) on
// v_mfma_scale_f32_16x16x128_f8f6f4.  A lane feeds 32 codes, 16 bytes, of one row and their scale byte; the products of codes and powers of two are
// exact, sums are in 32 bits.
#include "block4.h"
#include "grouped_kernels.h"

namespace lmk {

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

struct Linear4Args {
    const char *x;              // codes [rows][code_bytes(k)]
    const uint8_t *xs;          // scales [rows][scale_bytes(k)]
    const char *w;              // of block g from row g n on
    const uint8_t *ws;
    const float *bias;          // [blocks][n] or NULL
    const u32 *offsets;
    u32 blocks, rows, n, k;
    u32 relu;
    void *y;
    u64 ldy;
    u32 tiles, col_tiles;
};

// acc += w x: rows of w along the accumulator's registers (four a lane), rows of x along its lanes.  Format 4: e2m1
__device__ __forceinline__ f32x4 product4(i32x4 w, u32 ws, i32x4 x, u32 xs, f32x4 acc)
{
    const i32x8 a = __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1), b = __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, (int)ws, 0, (int)xs);
}

template <class T> __device__ __forceinline__ void finish(T *y, float v, u32 relu)
{
    if (relu) v = v < 0.0f ? 0.0f : v;                  // NaN stays
    *y = (T)v;
}

// ---- few rows: a workgroup takes 16 of them and NT outputs, its eight wavefronts share out the sum
constexpr u32 kRows = 16;

template <class T, u32 NT>
__global__ __launch_bounds__(512, 4) void few_rows4_kernel(const Linear4Args r)
{
    constexpr u32 kWaves = 8, kC = NT / 16, kAhead = NT == 64 ? 2 : 4;
    __shared__ float part[kWaves][kRows][NT + 1];
    const u32 row_tile = blockIdx.x / r.col_tiles, col0 = (blockIdx.x - row_tile * r.col_tiles) * NT;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kRows, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kRows;
    const u32 height = run.end - row0 < kRows ? run.end - row0 : kRows;
    const u32 width = r.n - col0 < NT ? r.n - col0 : NT;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 15, q = lane >> 4;
    const bool inside = run.block != ~0u;
    if (inside) {
        const u32 row_bytes = code_bytes(r.k), scales = scale_bytes(r.k), all = row_bytes / 64, per = (all + kWaves - 1) / kWaves;
        const u32 first = wave * per, last = first + per < all ? first + per : all;
        const u32 xrow = row0 + (j < height ? j : 0);
        const char *x = r.x + (u64)xrow * row_bytes + q * 16;
        const uint8_t *xs = r.xs + (u64)xrow * scales + q;
        u64 wrow[kC];
#pragma unroll
        for (u32 c = 0; c < kC; ++c) wrow[c] = (u64)run.block * r.n + col0 + (16 * c + j < width ? 16 * c + j : 0);
        f32x4 acc[kC] = {};
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
            i32x4 fx[kAhead], fw[kAhead][kC];
            u32 sx[kAhead], sw[kAhead][kC];
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                // a step that is not there is the first one again, and not multiplied
                const u32 t = t0 + a < last ? t0 + a : first;
                fx[a] = *reinterpret_cast<const i32x4 *>(x + t * 64);
                sx[a] = xs[t * 4];
#pragma unroll
                for (u32 c = 0; c < kC; ++c) {
                    fw[a][c] = *reinterpret_cast<const i32x4 *>(r.w + wrow[c] * row_bytes + q * 16 + t * 64);
                    sw[a][c] = r.ws[wrow[c] * scales + q + t * 4];
                }
            }
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                if (t0 + a >= last) break;
#pragma unroll
                for (u32 c = 0; c < kC; ++c) acc[c] = product4(fw[a][c], sw[a][c], fx[a], sx[a], acc[c]);
            }
        }
        // result c: outputs 16 c + 4 q .. + 3 of row j
#pragma unroll
        for (u32 c = 0; c < kC; ++c)
#pragma unroll
            for (u32 v = 0; v < 4; ++v) part[wave][j][16 * c + 4 * q + v] = acc[c][v];
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < kRows * NT; i += 512) {
        const u32 row = i / NT, c = i % NT;
        if (row >= height || c >= width) continue;
        float y = 0.0f;
        if (inside) {
#pragma unroll
            for (u32 p = 0; p < kWaves; ++p) y += part[p][row][c];
            if (r.bias) y += r.bias[(u64)run.block * r.n + col0 + c];
        }
        finish(static_cast<T *>(r.y) + (u64)(row0 + row) * r.ldy + col0 + c, y, r.relu);
    }
}

template <class T, u32 NT> hipError_t few_go(Linear4Args r, hipStream_t stream)
{
    r.col_tiles = (r.n + NT - 1) / NT;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kRows) * r.col_tiles);
    hipLaunchKernelGGL((few_rows4_kernel<T, NT>), dim3(r.tiles), dim3(512), 0, stream, r);
    return hipGetLastError();
}
u32 few_columns(const Linear4Args &r) { return max_runs(r.rows, r.blocks, kRows) * ((r.n + 63) / 64) >= 320 ? 64 : 16; }

Linear4Args linear4_args(const lmk_gs_linear4 &l, const lmk_gs_block4 &x, const float *bias, bool relu, void *y, u64 ldy)
{
    Linear4Args r = {};
    r.x = reinterpret_cast<const char *>(x.codes); r.xs = x.scale;
    r.w = reinterpret_cast<const char *>(l.w.codes); r.ws = l.w.scale;
    r.bias = bias;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.n = l.n; r.k = l.k;
    r.relu = relu;
    r.y = y; r.ldy = ldy;
    return r;
}

template <class T> hipError_t linear4_as(const Linear4Args &r, hipStream_t stream)
{
    return few_columns(r) == 64 ? few_go<T, 64>(r, stream) : few_go<T, 16>(r, stream);
}

}  // namespace

bool grouped_linear4_fits(const lmk_gs_linear4 &l)
{
    const Linear4Args r = linear4_args(l, {}, nullptr, false, nullptr, 0);
    const u32 nt = few_columns(r);
    return max_runs(r.rows, r.blocks, kRows) * ((r.n + nt - 1) / nt) * 512 < kMostThreads;
}

hipError_t launch_grouped_linear4(const lmk_gs_linear4 &l, const lmk_gs_block4 &x, const float *bias, bool relu, void *y, u64 ldy,
                                  hipStream_t stream)
{
    const Linear4Args r = linear4_args(l, x, bias, relu, y, ldy);
    return l.dtype == LMK_GS_F32 ? linear4_as<float>(r, stream) : linear4_as<__bf16>(r, stream);
}

}  // namespace lmk
