// What the kernels of gated layers share: the activation, its slope, and their arguments.
#ifndef LMK_GS_GROUPED_GATED_H
#define LMK_GS_GROUPED_GATED_H
#include "grouped_kernels.h"

namespace lmk {

// rows of a block against both projections of its weights
struct GatedArgs {
    const void *x;              // [rows][k]
    u64 ldx;
    const void *w;              // block g at g * w_block: [2 n][k] or [k][2 n], the gate's n first
    u64 ldw, w_block;
    const float *bias;          // [blocks][2 n] or NULL
    const u32 *offsets;
    u32 blocks, rows, n, k;
    u32 act;
    bool in_major;
    void *out;                  // y [rows][n], or the gradients of both projections [rows][2 n]
    u64 ldo;
    const void *dy;             // NULL: y is asked for
    u64 lddy;
    float *part;                // NULL, or sets of partial sums over rows of the gradients, 2 n each
    float *db;                  // where blocks of one set have theirs
    u32 tiles, col_tiles;
    bool out32;                 // gradients of few rows: in 32 bits whatever the type
    bool past;                  // `out` is more than the caches of the dies hold
};

// 1 / (1 + e^-a): the exponent's product is off by |a| 2^-24, which is e^-a's relative error
__device__ __forceinline__ float logistic(float a)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a * -1.44269504f));
}
// The normal distribution at a, and its density, each within 12 roundings of itself as long as it is 2^-126 or more; below that 0 for it.
// erfc(x) e^(x^2) / 2 of x = |a| / sqrt 2 is t P(t), t = 1 / (1 + p x), P of degree 8 with the least largest relative deviation over x up to 9.6
// (2.3e-8, by least squares with weights that grow where the deviation does).  -x^2 log2 e is taken in two parts: rounded once, the power of two of it
// would be off by a^2 2^-24 of itself.  From |a| = 16 on both are as they are there.
__device__ __forceinline__ float normal(float a, float &density)
{
    const float x = __builtin_fminf(__builtin_fabsf(a), 16.0f), q = x * x, rest = __builtin_fmaf(x, x, -q);
    constexpr float kHi = -0.72134752f, kLo = (float)(-0.72134752044448170368 - (double)kHi);          // -log2(e) / 2
    const float y = q * kHi, low = __builtin_fmaf(rest, kHi, __builtin_fmaf(q, kLo, __builtin_fmaf(q, kHi, -y)));
    float e = __builtin_amdgcn_exp2f(y);
    e = __builtin_fmaf(e, low * 0.69314718f, e);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.34648234f, x, 1.0f));
    float s = __builtin_fmaf(-0.028645312f, t, 0.145065382f);
    s = __builtin_fmaf(s, t, -0.266854078f);
    s = __builtin_fmaf(s, t, 0.178982466f);
    s = __builtin_fmaf(s, t, -0.0332354568f);
    s = __builtin_fmaf(s, t, 0.109878853f);
    s = __builtin_fmaf(s, t, 0.118032135f);
    s = __builtin_fmaf(s, t, 0.138562888f);
    s = __builtin_fmaf(s, t, 0.138213098f);
    const float tail = s * t * e;
    density = e * 0.398942280f;
    return a < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float gated(u32 act, float a, float u)
{
    if (act == LMK_GS_SILU) return a * logistic(a) * u;
    if (act == LMK_GS_RELU) return (a < 0.0f ? 0.0f : a) * u;           // NaN stays
    float density;
    return a * normal(a, density) * u;
}
// gradients of a and u from that of the product
__device__ __forceinline__ void gated_gradient(u32 act, float a, float u, float dy, float &da, float &du)
{
    if (act == LMK_GS_RELU) {
        da = a <= 0.0f ? 0.0f : dy * u;                                 // NaN lets it pass
        du = dy * (a < 0.0f ? 0.0f : a);
        return;
    }
    float p, slope;
    if (act == LMK_GS_SILU) {
        p = logistic(a);
        slope = p * (1.0f + a * (1.0f - p));
    } else {
        float density;
        p = normal(a, density);
        slope = p + a * density;
    }
    da = dy * u * slope;
    du = dy * (a * p);
}

// The set of run `local` of a block whose first row is `begin`, in runs of `per` rows, as launch_join numbers them
__device__ __forceinline__ float *set_of(const GatedArgs &r, const RowRun &run, u32 per)
{
    if (run.end - run.begin <= per) return r.db + (u64)run.block * 2 * r.n;
    RowSlices all;
    all.init(r.offsets, r.blocks, r.rows, per);
    return r.part + (u64)(run.block + all.slice_of(run.begin) + run.local) * 2 * r.n;
}

// `..._rows`: rows of a tile, which are those of a set of partial sums; `..._threads`: those that a launch would have
bool gated_few_fit(const GatedArgs &r, bool wide);
u64 gated_few_threads(const GatedArgs &r);
hipError_t launch_gated_few(const GatedArgs &r, u32 dtype, hipStream_t stream);
// all gradients of few rows, those of both projections in 32 bits in between: `grads` [rows][2 n], rows ldg apart, whole vectors
bool gated_few_backward_fits(u32 rows, u32 blocks, u32 n, u32 k, u32 dtype);
hipError_t launch_gated_few_backward(GatedArgs r, u32 dtype, float *grads, u64 ldg, void *dx, u64 lddx, void *dw, float *db, hipStream_t stream);
constexpr u32 kGatedFewRows = 16, kGatedTileRows = 64;

// small matrices, float32: y; all gradients in one pass, the sets of partial sums as launch_join numbers them, in runs of `.._backward_rows`
bool gated_narrow_fits(const GatedArgs &r);
u64 gated_narrow_threads(const GatedArgs &r);
hipError_t launch_gated_narrow(const GatedArgs &r, hipStream_t stream);
bool gated_narrow_backward_fits(const GatedArgs &r, u64 lddx);
u32 gated_narrow_backward_rows(const GatedArgs &r);
hipError_t launch_gated_narrow_backward(const GatedArgs &r, float *dx, u64 lddx, float *dw, float *db, float *part, hipStream_t stream);

bool gated_wide_fits(const GatedArgs &r);
u32 gated_wide_rows(const GatedArgs &r);
u64 gated_wide_threads(const GatedArgs &r);
hipError_t launch_gated_wide(const GatedArgs &r, hipStream_t stream);

}  // namespace lmk
#endif
