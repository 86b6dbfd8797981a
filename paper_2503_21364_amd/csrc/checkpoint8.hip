// 8-bit form of a layer's input, and back (lmk_gs_checkpoint8).  Bound by memory: one pass over the values,
// four consecutive ones a lane, so that the eight lanes of 32 values find their largest by exchanges inside
// the wavefront and a wavefront writes 256 codes in whole lines.  300 000 x 96 in float32 (144 MB either way): 35 us to the
// 8-bit form (4.1 TB/s), 22 us back (6.5 TB/s: the codes come from cache there).
#include "grouped.h"

namespace lmk {

namespace {

constexpr u32 kLanes = 8;                 // lanes of 32 values
constexpr u32 kPerBlock = 256 * 4;        // items (four values) of a workgroup

// Item numbers run through the padded rows; the first of a workgroup is divided once, in 64 bits.
struct ItemRow {
    u32 row, quad;
};
__device__ __forceinline__ ItemRow item_row(u32 row0, u32 quad0, u32 step, u32 quads)
{
    const u32 q = quad0 + step;
    const u32 r = q / quads;
    return ItemRow{row0 + r, q - r * quads};
}

template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const T *__restrict__ x, u64 ldx, u32 rows, u32 k,
                                                   const u32 *__restrict__ offsets, u32 blocks,
                                                   u32 *__restrict__ codes, uint8_t *__restrict__ scale)
{
    // with offsets, rows of no block are not read and kept as zeros
    const u32 lo = offsets ? offsets[0] : 0u, hi = offsets ? offsets[blocks] : rows;
    const u32 quads = (k + 31) / 32 * 8;
    const u64 first = (u64)blockIdx.x * kPerBlock;
    const u32 row0 = (u32)(first / quads), quad0 = (u32)(first - (u64)row0 * quads);
    f32x4 v[4];
    ItemRow at[4];
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        at[i] = item_row(row0, quad0, i * 256 + threadIdx.x, quads);
        v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (at[i].row >= rows || at[i].row < lo || at[i].row >= hi) continue;
        const u32 c = at[i].quad * 4;
        const T *p = x + (u64)at[i].row * ldx + c;
        if (c + 4 <= k) {
            v[i] = load4(p);
        } else {
#pragma unroll
            for (u32 j = 0; j < 4; ++j)
                if (c + j < k) v[i][j] = to_f32(p[j]);
        }
    }
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        u32 top = 0;
#pragma unroll
        for (u32 j = 0; j < 4; ++j) {
            const u32 b = __float_as_uint(v[i][j]) & 0x7fffffffu;
            top = top > b ? top : b;
        }
#pragma unroll
        for (u32 m = 1; m < kLanes; m *= 2) {
            const u32 other = (u32)__shfl_xor((int)top, (int)m, (int)kWave);
            top = top > other ? top : other;
        }
        if (at[i].row >= rows) continue;          // whole groups of eight lanes
        const u32 s = scale_of_max(top);
        const float inv = inverse_step(s);
        const u64 item = (u64)at[i].row * quads + at[i].quad;
        codes[item] = pack_codes(code_of(v[i][0], inv), code_of(v[i][1], inv), code_of(v[i][2], inv), code_of(v[i][3], inv));
        if ((threadIdx.x & (kLanes - 1)) == 0) scale[item / kLanes] = (uint8_t)s;
    }
}

template <class T>
__global__ __launch_bounds__(256) void unpack_kernel(const u32 *__restrict__ codes, const uint8_t *__restrict__ scale,
                                                     u32 rows, u32 k, T *__restrict__ x, u64 ldx)
{
    const u32 quads = (k + 31) / 32 * 8;
    const u64 first = (u64)blockIdx.x * kPerBlock;
    const u32 row0 = (u32)(first / quads), quad0 = (u32)(first - (u64)row0 * quads);
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        const ItemRow at = item_row(row0, quad0, i * 256 + threadIdx.x, quads);
        const u32 c = at.quad * 4;
        if (at.row >= rows || c >= k) continue;
        const u64 item = (u64)at.row * quads + at.quad;
        const u32 q = codes[item];
        const float step = step_of(scale[item / kLanes]);
        T *p = x + (u64)at.row * ldx + c;
        if (c + 4 <= k) {
            store4(p, f32x4{value_of(q, 0, step), value_of(q, 1, step), value_of(q, 2, step), value_of(q, 3, step)});
        } else {
#pragma unroll
            for (u32 j = 0; j < 4; ++j)
                if (c + j < k) p[j] = (T)value_of(q, j, step);
        }
    }
}

template <class T>
hipError_t pack_as(const void *x, u64 ldx, u32 rows, u32 k, const u32 *offsets, u32 blocks, const lmk_gs_checkpoint8 &out,
                   u32 grid, hipStream_t stream)
{
    hipLaunchKernelGGL(pack_kernel<T>, dim3(grid), dim3(256), 0, stream, (const T *)x, ldx, rows, k, offsets, blocks,
                       reinterpret_cast<u32 *>(out.codes), out.scale);
    return hipGetLastError();
}
template <class T>
hipError_t unpack_as(const lmk_gs_checkpoint8 &kept, u32 rows, u32 k, void *x, u64 ldx, u32 grid, hipStream_t stream)
{
    hipLaunchKernelGGL(unpack_kernel<T>, dim3(grid), dim3(256), 0, stream, reinterpret_cast<const u32 *>(kept.codes), kept.scale,
                       rows, k, (T *)x, ldx);
    return hipGetLastError();
}

}  // namespace

static u64 workgroups(u32 rows, u32 k) { return ((u64)rows * ((k + 31) / 32 * 8) + kPerBlock - 1) / kPerBlock; }

u64 checkpoint8_threads(u32 rows, u32 k) { return workgroups(rows, k) * 256; }

hipError_t launch_checkpoint8_pack(const void *x, u64 ldx, u32 rows, u32 k, u32 dtype, const u32 *offsets, u32 blocks,
                                   const lmk_gs_checkpoint8 &out, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const u32 grid = (u32)workgroups(rows, k);
    return dtype == LMK_GS_F32 ? pack_as<float>(x, ldx, rows, k, offsets, blocks, out, grid, stream)
                               : pack_as<__bf16>(x, ldx, rows, k, offsets, blocks, out, grid, stream);
}

hipError_t launch_checkpoint8_unpack(const lmk_gs_checkpoint8 &kept, u32 rows, u32 k, u32 dtype, void *x, u64 ldx,
                                     hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const u32 grid = (u32)workgroups(rows, k);
    return dtype == LMK_GS_F32 ? unpack_as<float>(kept, rows, k, x, ldx, grid, stream)
                               : unpack_as<__bf16>(kept, rows, k, x, ldx, grid, stream);
}

}  // namespace lmk
