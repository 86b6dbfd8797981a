// 4-bit form of a matrix, and back (lmk_gs_block4).  Bound by memory: one pass over the values, eight consecutive ones a lane, so that
// the four lanes of 32 values find their largest by exchanges inside the wavefront and a wavefront writes 512 codes in whole lines.
#include "block4.h"

namespace lmk {

namespace {

constexpr u32 kItem = 8;                    // values of a lane
constexpr u32 kPerBlock = 256 * 4;          // items of a workgroup

// Item numbers run through the rows; the first of a workgroup is divided once, in 64 bits.
struct ItemRow {
    u32 row, item;
};
__device__ __forceinline__ ItemRow item_row(u32 row0, u32 item0, u32 step, u32 items)
{
    const u32 q = item0 + step, r = q / items;
    return ItemRow{row0 + r, q - r * items};
}

typedef __attribute__((ext_vector_type(8))) float f32x8;
__device__ __forceinline__ f32x8 load8(const float *p) { return load_any<f32x8>(p); }
__device__ __forceinline__ f32x8 load8(const __bf16 *p)
{
    const bf16x8 v = load_any<bf16x8>(p);
    f32x8 o;
#pragma unroll
    for (u32 e = 0; e < 8; ++e) o[e] = (float)v[e];
    return o;
}

template <class T>
__global__ __launch_bounds__(256) void pack4_kernel(const T *__restrict__ x, u64 ldx, u32 rows, u32 k, u32 *__restrict__ codes,
                                                    uint8_t *__restrict__ scale)
{
    // a row of items is as long as its scales, four items each; what is beyond the codes has none
    const u32 items = scale_bytes(k) * 4, quads = code_bytes(k) / 4;
    const u64 first = (u64)blockIdx.x * kPerBlock;
    const u32 row0 = (u32)(first / items), item0 = (u32)(first - (u64)row0 * items);
    f32x8 v[4];
    ItemRow at[4];
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        at[i] = item_row(row0, item0, i * 256 + threadIdx.x, items);
        v[i] = f32x8{};
        if (at[i].row >= rows) continue;
        const u32 c = at[i].item * kItem;
        const T *p = x + (u64)at[i].row * ldx + c;
        if (c + kItem <= k) {
            v[i] = load8(p);
        } else {
#pragma unroll
            for (u32 j = 0; j < kItem; ++j)
                if (c + j < k) v[i][j] = to_f32(p[j]);
        }
    }
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        u32 top = 0;
#pragma unroll
        for (u32 j = 0; j < kItem; ++j) {
            const u32 b = __float_as_uint(v[i][j]) & 0x7fffffffu;
            top = top > b ? top : b;
        }
        u32 other = wave_dpp<0xB1, 0xf>(0u, top);           // lanes 1 0 3 2
        top = top > other ? top : other;
        other = wave_dpp<0x4E, 0xf>(0u, top);               // lanes 2 3 0 1
        top = top > other ? top : other;
        if (at[i].row >= rows) continue;                    // whole groups of four lanes
        const u32 s = scale4_of_max(top);
        const float inv = inverse_step(s);
        u32 o = 0;
#pragma unroll
        for (u32 j = 0; j < kItem; ++j) o |= code4_of(v[i][j], inv) << (4 * j);
        if (s == 0u || s == 255u) o = s == 0u ? o : 0u;
        if (at[i].item < quads) codes[(u64)at[i].row * quads + at[i].item] = o;
        if ((threadIdx.x & 3) == 0) scale[(u64)at[i].row * (items / 4) + at[i].item / 4] = (uint8_t)s;
    }
}

template <class T>
__global__ __launch_bounds__(256) void unpack4_kernel(const u32 *__restrict__ codes, const uint8_t *__restrict__ scale, u32 rows, u32 k,
                                                      T *__restrict__ x, u64 ldx)
{
    const u32 quads = code_bytes(k) / 4, items = (k + kItem - 1) / kItem;
    const u64 first = (u64)blockIdx.x * kPerBlock;
    const u32 row0 = (u32)(first / items), item0 = (u32)(first - (u64)row0 * items);
#pragma unroll
    for (u32 i = 0; i < 4; ++i) {
        const ItemRow at = item_row(row0, item0, i * 256 + threadIdx.x, items);
        if (at.row >= rows) continue;
        const u32 c = at.item * kItem, q = codes[(u64)at.row * quads + at.item];
        const float step = step_of(scale[(u64)at.row * scale_bytes(k) + at.item / 4]);
        T *p = x + (u64)at.row * ldx + c;
        f32x8 v;
#pragma unroll
        for (u32 j = 0; j < kItem; ++j) v[j] = value4_of(q >> (4 * j), step);
        if (c + kItem <= k) {
            store_any(p, __builtin_convertvector(v, T __attribute__((ext_vector_type(8)))));
        } else {
#pragma unroll
            for (u32 j = 0; j < kItem; ++j)
                if (c + j < k) p[j] = (T)v[j];
        }
    }
}

u64 pack_workgroups(u32 rows, u32 k) { return ((u64)rows * scale_bytes(k) * 4 + kPerBlock - 1) / kPerBlock; }
u64 unpack_workgroups(u32 rows, u32 k) { return ((u64)rows * ((k + kItem - 1) / kItem) + kPerBlock - 1) / kPerBlock; }

}  // namespace

// the larger of the two
u64 block4_threads(u32 rows, u32 k) { return pack_workgroups(rows, k) * 256; }

hipError_t launch_block4_pack(const void *x, u64 ldx, u32 rows, u32 k, u32 dtype, const lmk_gs_block4 &out, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const dim3 grid((u32)pack_workgroups(rows, k));
    u32 *codes = reinterpret_cast<u32 *>(out.codes);
    if (dtype == LMK_GS_F32) hipLaunchKernelGGL(pack4_kernel<float>, grid, dim3(256), 0, stream, (const float *)x, ldx, rows, k, codes, out.scale);
    else hipLaunchKernelGGL(pack4_kernel<__bf16>, grid, dim3(256), 0, stream, (const __bf16 *)x, ldx, rows, k, codes, out.scale);
    return hipGetLastError();
}

hipError_t launch_block4_unpack(const lmk_gs_block4 &form, u32 rows, u32 k, u32 dtype, void *x, u64 ldx, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const dim3 grid((u32)unpack_workgroups(rows, k));
    const u32 *codes = reinterpret_cast<const u32 *>(form.codes);
    if (dtype == LMK_GS_F32) hipLaunchKernelGGL(unpack4_kernel<float>, grid, dim3(256), 0, stream, codes, form.scale, rows, k, (float *)x, ldx);
    else hipLaunchKernelGGL(unpack4_kernel<__bf16>, grid, dim3(256), 0, stream, codes, form.scale, rows, k, (__bf16 *)x, ldx);
    return hipGetLastError();
}

}  // namespace lmk
