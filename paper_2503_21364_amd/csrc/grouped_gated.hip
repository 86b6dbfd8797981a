// Gated layers whose weights belong to blocks of rows (lmk_gs_grouped_gated): y = act(x Wg^T + bg) * (x Wu^T + bu), both projections, the
// activation and the product in one kernel, and the gradients.  Here: the choice of kernels, and the one that takes every size, stride,
// alignment and type.
//
// The gradients keep nothing of the forward pass: a kernel takes both projections again and writes their gradients
//     da = dy u act'(a),  du = dy act(a)
// side by side, [rows][2 n], in the workspace; from there dx = [da du] W and dW = [da du]^T x are the grouped layers' own products.
// In bfloat16 da and du are rounded there: the matrix instructions take nothing wider, and two bfloat16 for each would be twice the products of dx
// and dW (some 900 us more at 16 384 rows of 2048 -> 4096 in 4 blocks, now 1500).  It costs as much as the results' own rounding (2.3e-3 altogether, without
// it 1.7e-3).  dW has the weights' type, half the bytes of 32 bits; who adds up many calls' adds in float32.  The bias' gradient does not go through them: it is summed in 32 bits beside the
// activation, before the rounding.  Few rows (grouped_gated_few.hip) and small float32 matrices (grouped_gated_narrow.hip) have da and du in 32 bits.
//
// Kernel here: v_mfma_f32_32x32x2_f32, tiles of 64 rows x 64 outputs of both projections, the rows' part of LDS being read for both.  Bound by
// those instructions where k is large; 25 362 rows, 64 -> 576: 62 us, 60 of 154 TFLOP/s, a tile being two steps between a chain of loads and its stores.
#include "grouped_gated.h"
#include "grouped_tiles.h"

namespace lmk {

namespace {

template <class T, bool ACROSS, bool BACKWARD>
__global__ __launch_bounds__(256, 3) void gated_rows_kernel(const GatedArgs r)
{
    constexpr u32 pitch = pitch_of(kTile), buffer = 3 * kStep * pitch;
    __shared__ __align__(16) float lds[2 * buffer];
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, 3 * kUnits);
    const u32 row_tile = tile / r.col_tiles, col0 = (tile - row_tile * r.col_tiles) * kTile;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kTile, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kTile;
    const u32 height = run.end - row0 < kTile ? run.end - row0 : kTile;
    const u32 width = r.n - col0 < kTile ? r.n - col0 : kTile;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 31, hi = lane / 32;
    const u32 m0 = wave / 2 * 32 + j, n0 = wave % 2 * 32 + j;
    const bool inside = run.block != ~0u;
    f32x16 acc[2] = {};
    if (inside) {
        using B = typename std::conditional<ACROSS, Across<T, kTile>, Along<T, kTile>>::type;
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        const u64 first = ACROSS ? col0 : (u64)col0 * r.ldw, second = ACROSS ? r.n + col0 : (u64)(r.n + col0) * r.ldw;
        Along<T, kTile> a{static_cast<const T *>(r.x) + (u64)row0 * r.ldx, r.ldx, height, r.k, {}};
        B bg{w + first, r.ldw, width, r.k, {}}, bu{w + second, r.ldw, width, r.k, {}};
        a.load(0);
        bg.load(0);
        bu.load(0);
        u32 at = 0;
        for (u32 s0 = 0; s0 < r.k; s0 += kStep, at ^= 1) {
            float *la = lds + at * buffer, *lg = la + kStep * pitch, *lu = lg + kStep * pitch;
            a.store(la);
            bg.store(lg);
            bu.store(lu);
            __syncthreads();                     // the other buffer's readers are past the previous one of these
            if (s0 + kStep < r.k) {
                a.load(s0 + kStep);
                bg.load(s0 + kStep);
                bu.load(s0 + kStep);
            }
            const u32 left = r.k - s0;
            auto step = [&](u32 t) {
                const u32 s = (t + 16 * hi) * pitch;
                const float v = la[s + m0];
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, lg[s + n0], acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, lu[s + n0], acc[1], 0, 0, 0);
            };
            if (left >= 16) {
#pragma unroll
                for (u32 t = 0; t < 16; ++t) step(t);
            } else {
                for (u32 t = 0; t < left; ++t) step(t);
            }
        }
    }
    const u32 c = wave % 2 * 32 + j;
    float bias[2] = {0.0f, 0.0f}, sum[2] = {0.0f, 0.0f};
    if (r.bias && inside && c < width) {
        const float *b = r.bias + (u64)run.block * 2 * r.n + col0 + c;
        bias[0] = b[0];
        bias[1] = b[r.n];
    }
    T *out = static_cast<T *>(r.out) + (u64)row0 * r.ldo + col0 + c;
#pragma unroll
    for (u32 v = 0; v < 16; ++v) {
        const u32 row = wave / 2 * 32 + row_of(v, hi);
        if (row >= height || c >= width) continue;
        const float a = acc[0][v] + bias[0], u = acc[1][v] + bias[1];
        if constexpr (!BACKWARD) {
            out[(u64)row * r.ldo] = (T)(inside ? gated(r.act, a, u) : 0.0f);
        } else {
            float da = 0.0f, du = 0.0f;
            if (inside) gated_gradient(r.act, a, u, to_f32(static_cast<const T *>(r.dy)[(u64)(row0 + row) * r.lddy + col0 + c]), da, du);
            out[(u64)row * r.ldo] = (T)da;
            out[(u64)row * r.ldo + r.n] = (T)du;
            sum[0] += da;
            sum[1] += du;
        }
    }
    if constexpr (BACKWARD) {
        if (!r.part || !inside) return;                 // the whole workgroup
        // rows of a column: in the lanes j and j + 32 of the two wavefronts below each other
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < 2; ++h) lds[(wave / 2 * 2 + hi) * 2 * kTile + h * kTile + c] = sum[h];
        __syncthreads();
        const u32 col = threadIdx.x % kTile, h = threadIdx.x / kTile;
        if (h >= 2 || col >= width) return;
        float s = 0.0f;
#pragma unroll
        for (u32 i = 0; i < 4; ++i) s += lds[i * 2 * kTile + h * kTile + col];
        set_of(r, run, kTile)[h * r.n + col0 + col] = s;
    }
}

template <class T>
hipError_t all_go(GatedArgs r, hipStream_t stream)
{
    r.col_tiles = (r.n + kTile - 1) / kTile;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kTile) * r.col_tiles);
    auto kernel = r.dy ? (r.in_major ? gated_rows_kernel<T, true, true> : gated_rows_kernel<T, false, true>)
                       : (r.in_major ? gated_rows_kernel<T, true, false> : gated_rows_kernel<T, false, false>);
    hipLaunchKernelGGL(kernel, dim3(r.tiles), dim3(kThreads), 0, stream, r);
    return hipGetLastError();
}

enum class GatedKernel { few, wide, narrow, all };
GatedKernel gated_choice(const GatedArgs &r, u32 dtype)
{
    const bool wide = dtype == LMK_GS_BF16 && gated_wide_fits(r), narrow = dtype == LMK_GS_F32 && !r.dy && gated_narrow_fits(r);
    return gated_few_fit(r, wide) ? GatedKernel::few : wide ? GatedKernel::wide : narrow ? GatedKernel::narrow : GatedKernel::all;
}
u64 gated_threads(const GatedArgs &r, u32 dtype)
{
    switch (gated_choice(r, dtype)) {
    case GatedKernel::few: return gated_few_threads(r);
    case GatedKernel::wide: return gated_wide_threads(r);
    case GatedKernel::narrow: return gated_narrow_threads(r);
    default: return max_runs(r.rows, r.blocks, kTile) * ((r.n + kTile - 1) / kTile) * kThreads;
    }
}
hipError_t gated_go(const GatedArgs &r, u32 dtype, hipStream_t stream)
{
    switch (gated_choice(r, dtype)) {
    case GatedKernel::few: return launch_gated_few(r, dtype, stream);
    case GatedKernel::wide: return launch_gated_wide(r, stream);
    case GatedKernel::narrow: return launch_gated_narrow(r, stream);
    default: return dtype == LMK_GS_F32 ? all_go<float>(r, stream) : all_go<__bf16>(r, stream);
    }
}
// rows of a set of partial sums of the bias' gradient
u32 gated_set_rows(const GatedArgs &r, u32 dtype)
{
    switch (gated_choice(r, dtype)) {
    case GatedKernel::few: return kGatedFewRows;
    case GatedKernel::wide: return gated_wide_rows(r);
    default: return kTile;
    }
}
static_assert(kTile == kGatedTileRows, "rows of a tile");

GatedArgs gated_args(const lmk_gs_linear &l, const void *x, u64 ldx, const float *bias, u32 act)
{
    GatedArgs r = {};
    r.x = x; r.ldx = ldx;
    r.w = l.w; r.ldw = l.ldw; r.w_block = l.w_block; r.in_major = l.in_major != 0;
    r.bias = bias;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.n = l.n; r.k = l.k;
    r.act = act;
    return r;
}

// both projections as one layer
lmk_gs_linear both(const lmk_gs_linear &l)
{
    lmk_gs_linear b = l;
    b.n = 2 * l.n;
    return b;
}
// all gradients in one kernel; dy of packed rows stands for any that fits
bool one_pass_fits(const GatedArgs &r, u32 dtype, u64 lddx) { return dtype == LMK_GS_F32 && gated_narrow_backward_fits(r, lddx); }
u64 round_up(u64 bytes) { return (bytes + 255) / 256 * 256; }
// elements between rows of both projections' gradients: whole vectors
u64 grads_stride(const lmk_gs_linear &l) { return ((u64)2 * l.n + 7) / 8 * 8; }

// Workspace: the gradients of both projections; partial sums of the bias' gradient where they are not the linear layer's; its own
struct GatedSpace {
    u64 grads, sums, linear;
};
GatedSpace gated_space(const lmk_gs_linear &l)
{
    GatedSpace s;
    const bool few = gated_few_backward_fits(l.rows, l.blocks, l.n, l.k, l.dtype);
    s.grads = round_up(l.rows * grads_stride(l) * (l.dtype == LMK_GS_F32 || few ? 4 : 2));
    // the least rows of a set that any alignment gives
    const GatedArgs r = gated_args(l, nullptr, l.k, nullptr, 0);
    const u32 least = gated_few_fit(r, false) || gated_few_fit(r, true) ? kGatedFewRows : kGatedTileRows;
    s.sums = l.dtype == LMK_GS_F32 ? 0 : round_up(((u64)l.rows / least + l.blocks + 1) * 2 * l.n * 4);
    s.linear = grouped_backward_bytes(both(l));
    if (one_pass_fits(r, l.dtype, l.k)) {
        const u64 sets = ((u64)l.rows / gated_narrow_backward_rows(r) + 1 + l.blocks) * ((u64)2 * l.n * l.k + 2 * l.n) * 4;
        s.linear = sets > s.linear ? sets : s.linear;
    }
    return s;
}

}  // namespace

bool grouped_gated_fits(const lmk_gs_linear &l, const void *x, u64 ldx, u64 ldy)
{
    GatedArgs r = gated_args(l, x, ldx, nullptr, 0);
    r.ldo = ldy;
    return gated_threads(r, l.dtype) < kMostThreads;
}

size_t grouped_gated_backward_bytes(const lmk_gs_linear &l)
{
    const GatedSpace s = gated_space(l);
    return (size_t)(s.grads + s.sums + s.linear);
}

bool grouped_gated_backward_fits(const lmk_gs_linear &l, u64 lddy, const void *x, u64 ldx, const lmk_gs_gated_grads &out)
{
    const bool own_db = l.dtype == LMK_GS_BF16 && out.db;
    GatedArgs r = gated_args(l, x, ldx, nullptr, 0);
    r.dy = reinterpret_cast<const void *>(256);             // told from NULL: gradients are asked for
    r.lddy = lddy;
    // one run a workgroup there, of which there are some hundred and one a block
    if (one_pass_fits(r, l.dtype, out.lddx)) return join_threads(2 * l.n, l.k, l.blocks, l.rows / gated_narrow_backward_rows(r) + 1) < kMostThreads;
    if (gated_few_backward_fits(l.rows, l.blocks, l.n, l.k, l.dtype)) return true;
    if (own_db && join_threads(2 * l.n, 0, l.blocks, l.rows / gated_set_rows(r, l.dtype) + 1) >= kMostThreads) return false;
    const lmk_gs_linear_grads grads = {out.dx, out.lddx, static_cast<float *>(out.dw), own_db ? nullptr : out.db};
    if (gated_threads(r, l.dtype) >= kMostThreads) return false;
    // the gradients' place in the workspace is aligned: any pointer that is stands for it
    return grouped_backward_fits(both(l), reinterpret_cast<const void *>(256), grads_stride(l), x, ldx, nullptr, false, grads);
}

hipError_t launch_grouped_gated(const lmk_gs_linear &l, const void *x, u64 ldx, const float *bias, u32 act, void *y, u64 ldy, hipStream_t stream)
{
    GatedArgs r = gated_args(l, x, ldx, bias, act);
    r.out = y;
    r.ldo = ldy;
    return gated_go(r, l.dtype, stream);
}

hipError_t launch_grouped_gated_backward(const lmk_gs_linear &l, const void *dy, u64 lddy, const void *x, u64 ldx, const float *bias, u32 act,
                                         const lmk_gs_gated_grads &out, char *workspace, hipStream_t stream)
{
    const GatedSpace space = gated_space(l);
    const bool own_db = l.dtype == LMK_GS_BF16 && out.db;
    GatedArgs r = gated_args(l, x, ldx, bias, act);
    r.dy = dy;
    r.lddy = lddy;
    char *linear_space = workspace + space.grads + space.sums;
    if (one_pass_fits(r, l.dtype, out.lddx)) {
        float *part = reinterpret_cast<float *>(linear_space), *dw = static_cast<float *>(out.dw);
        const hipError_t e = launch_gated_narrow_backward(r, static_cast<float *>(out.dx), out.lddx, dw, out.db, part, stream);
        if (e != hipSuccess || !(dw || out.db)) return e;
        const u32 per = gated_narrow_backward_rows(r);
        return launch_join(l.offsets, l.blocks, l.rows, per, part, 2 * l.n, l.k, dw, out.db, l.rows / per + 1, stream);
    }
    if (gated_few_backward_fits(l.rows, l.blocks, l.n, l.k, l.dtype))
        return launch_gated_few_backward(r, l.dtype, reinterpret_cast<float *>(workspace), grads_stride(l), out.dx, out.lddx, out.dw, out.db, stream);
    r.out = workspace;
    r.ldo = grads_stride(l);
    if (own_db) {
        r.part = reinterpret_cast<float *>(workspace + space.grads);
        r.db = out.db;
    }
    hipError_t e = hipSuccess;
    if (l.rows > 0) e = gated_go(r, l.dtype, stream);
    if (e == hipSuccess && own_db) {
        const u32 per = gated_set_rows(r, l.dtype);
        e = launch_join(l.offsets, l.blocks, l.rows, per, r.part, 2 * l.n, 0, nullptr, out.db, l.rows / per + 1, stream);
    }
    if (e != hipSuccess || !(out.dx || out.dw || (out.db && !own_db))) return e;
    const lmk_gs_linear_grads grads = {out.dx, out.lddx, static_cast<float *>(out.dw), own_db ? nullptr : out.db};
    return launch_grouped_backward(both(l), workspace, grads_stride(l), x, ldx, nullptr, false, grads, linear_space, stream,
                                   l.dtype == LMK_GS_BF16);
}

}  // namespace lmk
