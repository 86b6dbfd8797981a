// Perceptron layers whose weights belong to blocks of rows (lmk_gs_grouped_linear and its gradients): the choice of
// kernels, the kernels that take every size, stride, alignment and type, and the one that joins partial sums.  Three
// products, of which the first two are one kernel:
//     y  = x w_g^T         rows of a block against the block's weights, sum over the inputs
//     dx = dy w_g          the same with the weights the other way round, sum over the outputs
//     dw_g = dy^T x        sum over the rows of a block
// Float32 matrix instructions (v_mfma_f32_32x32x2_f32: products and sums in 32 bits); bfloat16 operands are widened
// while they are staged, which is exact.
//
// Bound by the rate of that instruction (154 TFLOP/s is what the largest library product reaches): 102 - 106 TFLOP/s at
// 8192 rows x 4096 x 4096, 84 at 65 536 x 256 x 256 in 32 blocks.
//
// Both operands of a tile pass through LDS as [sum index][row or column]: a lane of half `hi` feeds sum
// index t + 16 hi to step t, so the 32 lanes of a half read 32 consecutive floats, and with a pitch of 66
// floats the two halves (16 pitches apart) are on different banks, as are the stores of an operand whose
// sum index is contiguous in memory (eight lanes along it, 8 banks apart; eight rows on the banks between).
#include "grouped_kernels.h"

namespace lmk {

namespace {

constexpr u32 kStep = 32;                 // sum indices of a staged step
constexpr u32 kThreads = 256;

constexpr u32 pitch_of(u32 width) { return width + 2; }

// ---- operands: how a tile of `W` rows (columns) by kStep sum indices comes from memory.  load() only
// requests; store() puts it into LDS.  Out of range: zeros.

// sum index contiguous in memory: element (m, s) at p[m * ld + s]
template <class T, u32 W> struct Along {
    const T *p;
    u64 ld;
    u32 width, sums;        // valid rows, valid sum indices
    float v[W / 8];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, m = c / 8, s = s0 + c % 8 * 4;
            f32x4 q = {0.f, 0.f, 0.f, 0.f};
            if (m < width) {
                const T *a = p + (u64)m * ld + s;
                if (s + 4 <= sums) q = load4(a);
                else {
#pragma unroll
                    for (u32 j = 0; j < 4; ++j)
                        if (s + j < sums) q[j] = to_f32(a[j]);
                }
            }
#pragma unroll
            for (u32 j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, m = c / 8, s = c % 8 * 4;
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[(s + j) * pitch + m] = v[4 * i + j];
        }
    }
};

// rows (columns) contiguous in memory: element (m, s) at p[s * ld + m]
template <class T, u32 W> struct Across {
    const T *p;
    u64 ld;
    u32 width, sums;
    float v[W / 8];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = s0 + c / (W / 4), m = c % (W / 4) * 4;
            f32x4 q = {0.f, 0.f, 0.f, 0.f};
            if (s < sums && m < width) {
                const T *a = p + (u64)s * ld + m;
                if (m + 4 <= width) q = load4(a);
                else {
#pragma unroll
                    for (u32 j = 0; j < 4; ++j)
                        if (m + j < width) q[j] = to_f32(a[j]);
                }
            }
#pragma unroll
            for (u32 j = 0; j < 4; ++j) v[4 * i + j] = q[j];
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = c / (W / 4), m = c % (W / 4) * 4;
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[s * pitch + m + j] = v[4 * i + j];
        }
    }
};

// the same from the 8-bit form: rows of kp codes (all of them there), a scale byte for 32
template <u32 W> struct Across8 {
    const u32 *codes;       // of the tile's first row and column
    const uint8_t *scale;
    u32 kp;                 // codes of a row
    u32 width, sums;        // width: codes to the end of the row
    u32 q[W / 32];
    u32 e[W / 32];

    __device__ __forceinline__ void load(u32 s0)
    {
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = s0 + c / (W / 4), m = c % (W / 4) * 4;
            const bool there = s < sums && m < width;
            q[i] = there ? codes[((u64)s * kp + m) / 4] : 0u;
            e[i] = there ? scale[(u64)s * (kp / 32) + m / 32] : 0u;
        }
    }
    __device__ __forceinline__ void store(float *lds) const
    {
        constexpr u32 pitch = pitch_of(W);
#pragma unroll
        for (u32 i = 0; i < W / 32; ++i) {
            const u32 c = threadIdx.x + i * kThreads, s = c / (W / 4), m = c % (W / 4) * 4;
            const float step = step_of(e[i]);
#pragma unroll
            for (u32 j = 0; j < 4; ++j) lds[s * pitch + m + j] = value_of(q[i], j, step);
        }
    }
};

// Tiles of 64 x 64 results, 32 x 32 a wavefront: four workgroups a compute unit hide what a step waits for, and the
// operands' way through LDS is no limit at this instruction's rate (128 x 128 tiles, two workgroups: 66 instead of 80 TFLOP/s at
// 65 536 x 256 x 256, 101 instead of 104 at 8192 x 4096 x 4096).
constexpr u32 kTile = 64;

// The product of a tile: acc += A B over `sums`.  `each` is called with the staged A of every step.
template <class A, class B, class Each>
__device__ __forceinline__ void tile_product(A &a, B &b, u32 sums, float *lds, f32x16 &acc, Each &&each)
{
    constexpr u32 pitch = pitch_of(kTile), buffer = 2 * kStep * pitch;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const u32 j = lane & 31, hi = lane / 32, m0 = wave / 2 * 32 + j, n0 = wave % 2 * 32 + j;
    a.load(0);
    b.load(0);
    u32 at = 0;
    for (u32 s0 = 0; s0 < sums; s0 += kStep, at ^= 1) {
        float *la = lds + at * buffer, *lb = la + kStep * pitch;
        a.store(la);
        b.store(lb);
        __syncthreads();                     // the other buffer's readers are past the previous one of these
        if (s0 + kStep < sums) {
            a.load(s0 + kStep);
            b.load(s0 + kStep);
        }
        each(la);
        // steps t and t + 16 in one instruction; the last ones of a short tile hold nothing
        const u32 left = sums - s0;
        auto step = [&](u32 t) {
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(la[(t + 16 * hi) * pitch + m0], lb[(t + 16 * hi) * pitch + n0], acc, 0, 0, 0);
        };
        if (left >= 16) {
#pragma unroll
            for (u32 t = 0; t < 16; ++t) step(t);
        } else {
            for (u32 t = 0; t < left; ++t) step(t);
        }
    }
}

// row of a 32 x 32 result that register v of a lane of half hi holds (its column is lane % 32)
__device__ __forceinline__ u32 row_of(u32 v, u32 hi) { return 8 * (v / 4) + 4 * hi + v % 4; }

// ---- rows against weights

// GATE: 0 none, 1 values, 2 codes
template <class T, bool ACROSS, u32 GATE>
__global__ __launch_bounds__(256, 4) void rows_kernel(const RowsArgs r)
{
    __shared__ __align__(16) float lds[4 * kStep * pitch_of(kTile)];
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, 4 * kUnits);
    const u32 row_tile = tile / r.col_tiles, col0 = (tile - row_tile * r.col_tiles) * kTile;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kTile, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kTile;
    const u32 height = run.end - row0 < kTile ? run.end - row0 : kTile;
    const u32 width = r.cols - col0 < kTile ? r.cols - col0 : kTile;
    T *out = static_cast<T *>(r.out) + (u64)row0 * r.ldo + col0;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 31, hi = lane / 32;
    f32x16 acc = {};
    if (run.block != ~0u) {
        Along<T, kTile> a{static_cast<const T *>(r.a) + (u64)row0 * r.lda, r.lda, height, r.sums, {}};
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        if constexpr (ACROSS) {
            Across<T, kTile> b{w + col0, r.ldw, width, r.sums, {}};
            tile_product(a, b, r.sums, lds, acc, [](const float *) {});
        } else {
            Along<T, kTile> b{w + (u64)col0 * r.ldw, r.ldw, width, r.sums, {}};
            tile_product(a, b, r.sums, lds, acc, [](const float *) {});
        }
    }
    const u32 c = wave % 2 * 32 + j;
    const float bias = (r.bias && run.block != ~0u && c < width) ? r.bias[(u64)run.block * r.cols + col0 + c] : 0.0f;
#pragma unroll
    for (u32 v = 0; v < 16; ++v) {
        const u32 row = wave / 2 * 32 + row_of(v, hi);
        if (row >= height || c >= width) continue;
        float y = acc[v] + bias;
        if (r.relu) y = y < 0.0f ? 0.0f : y;              // NaN stays
        if (GATE == 1 && run.block != ~0u) {
            const float x = to_f32(static_cast<const T *>(r.gate)[(u64)(row0 + row) * r.ldgate + col0 + c]);
            y = x <= 0.0f ? 0.0f : y;
        }
        if (GATE == 2 && run.block != ~0u) {
            const u64 at = (u64)(row0 + row) * r.ldgate + col0 + c;
            const bool pass = static_cast<const signed char *>(r.gate)[at] > 0 || r.gate_scale[at / 32] == 255;
            y = pass ? y : 0.0f;
        }
        out[(u64)row * r.ldo + c] = (T)y;
    }
}

// ---- sums over the rows of a block

// KIND: 0 no x (db alone), 1 values, 2 codes
template <class T, u32 KIND>
__global__ __launch_bounds__(256, 4) void sums_kernel(const SumsArgs r)
{
    __shared__ __align__(16) float lds[4 * kStep * pitch_of(kTile)];
    const u32 tile = tile_of_workgroup(blockIdx.x, r.tiles, 4 * kUnits);
    const u32 pairs = r.n_tiles * r.k_tiles, slice = tile / pairs, pair = tile - slice * pairs;
    const u32 n0 = pair / r.k_tiles * kTile, k0 = pair % r.k_tiles * kTile;
    const u32 height = r.n - n0 < kTile ? r.n - n0 : kTile, width = r.k - k0 < kTile ? r.k - k0 : kTile;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 31, hi = lane / 32;
    SliceRuns run;
    run.init(r.offsets, r.blocks, r.rows, r.per, slice);
    while (run.next()) {
        f32x16 acc = {};
        float bias = 0.0f;
        __syncthreads();                    // the run in front of this one is out of LDS
        Across<T, kTile> a{static_cast<const T *>(r.dy) + (u64)run.row * r.lddy + n0, r.lddy, height, run.count, {}};
        // thread m sums column m of the staged dy
        const bool sums_db = r.db && k0 == 0 && threadIdx.x < kTile;
        auto each = [&](const float *la) {
            if (!sums_db) return;
#pragma unroll
            for (u32 s = 0; s < kStep; ++s) bias += la[s * pitch_of(kTile) + threadIdx.x];
        };
        if constexpr (KIND == 2) {
            const u32 kp = (r.k + 31) / 32 * 32;
            Across8<kTile> b{reinterpret_cast<const u32 *>(static_cast<const signed char *>(r.x) + (u64)run.row * kp + k0),
                             r.scale + ((u64)run.row * kp + k0) / 32, kp, kp - k0, run.count, {}, {}};
            tile_product(a, b, run.count, lds, acc, each);
        } else {
            Across<T, kTile> b{static_cast<const T *>(r.x) + (KIND == 1 ? (u64)run.row * r.ldx + k0 : 0), r.ldx, KIND == 1 ? width : 0u,
                               run.count, {}};
            tile_product(a, b, run.count, lds, acc, each);
        }
        const u64 size = (u64)r.n * r.k;
        float *dw = run.whole ? r.dw + (u64)run.block * size : r.part + (u64)run.partial() * (size + r.n);
        float *db = run.whole ? r.db + (u64)run.block * r.n : r.part + (u64)run.partial() * (size + r.n) + size;
        if (r.dw) {
            const u32 col = wave % 2 * 32 + j;
#pragma unroll
            for (u32 v = 0; v < 16; ++v) {
                const u32 row = wave / 2 * 32 + row_of(v, hi);
                if (row >= height || col >= width) continue;
                dw[r.in_major ? (u64)(k0 + col) * r.n + n0 + row : (u64)(n0 + row) * r.k + k0 + col] = acc[v];
            }
        }
        if (r.db && k0 == 0 && threadIdx.x < height) db[n0 + threadIdx.x] = bias;
    }
}

// Joins the partial sums of the blocks that have several runs, in the order of the runs (the same bits every time), and
// writes zeros for blocks without rows.  V consecutive sums a thread, AHEAD sets on their way: no sum waits for the one in
// front of it, only its addition does.  Where there are few sums, and so many sets of them, PARTS parts of a workgroup take
// consecutive sets each and the parts meet in LDS, in their order.  Bound by memory where there are many sums (32 blocks of 1024 x 1024: 37 us), by
// the chain of sets where there are few.
template <u32 V, u32 AHEAD, u32 PARTS>
__global__ __launch_bounds__(256) void join_kernel(const u32 *__restrict__ offsets, u32 blocks, u32 rows, u32 per, bool by_blocks,
                                                   const float *__restrict__ part, u32 n, u32 k, float *__restrict__ dw,
                                                   float *__restrict__ db, u32 pieces)
{
    typedef __attribute__((ext_vector_type(V))) float vec;
    constexpr u32 kWidth = 256 / PARTS;                 // threads along the sums
    const u32 block = blockIdx.x / pieces, piece = blockIdx.x - block * pieces;
    RowSlices all;
    all.init(offsets, blocks, rows, per);
    u32 b, e;
    all.block(block, b, e);
    // no runs: zeros; one: written where it was summed
    const u32 first = all.slice_of(b), runs = b == e ? 0u : by_blocks ? (e - b + per - 1) / per : all.slice_of(e - 1) - first + 1;
    if (runs == 1) return;
    const u64 size = (u64)n * k, stride = size + n;
    const float *p = part + (u64)(first + block) * stride;
    const u32 share = (runs + PARTS - 1) / PARTS, part_of = threadIdx.x / kWidth;
    const u32 from = part_of * share, to = from + share < runs ? from + share : runs;
    const auto sum = [&](auto zero, u64 at) {
        auto s = zero;
        for (u32 q = from; q < to; q += AHEAD) {
            decltype(zero) v[AHEAD];
#pragma unroll
            for (u32 h = 0; h < AHEAD; ++h) v[h] = load_any<decltype(zero)>(p + (u64)(q + h < to ? q + h : q) * stride + at);
#pragma unroll
            for (u32 h = 0; h < AHEAD; ++h)
                if (q + h < to) s += v[h];
        }
        return s;
    };
    const u64 at = ((u64)piece * kWidth + threadIdx.x % kWidth) * V;
    if constexpr (PARTS > 1) {
        static_assert(V == 1, "a thread of each part for a sum");
        __shared__ float parts[PARTS][kWidth];
        const bool there = at < stride && (at < size ? dw != nullptr : db != nullptr);
        parts[part_of][threadIdx.x % kWidth] = there ? sum(0.0f, at) : 0.0f;
        __syncthreads();
        if (part_of != 0 || !there) return;
        float s = 0.0f;
#pragma unroll
        for (u32 q = 0; q < PARTS; ++q) s += parts[q][threadIdx.x];
        (at < size ? dw[(u64)block * size + at] : db[(u64)block * n + (at - size)]) = s;
        return;
    }
    if (V > 1 && at + V <= size) {
        if (dw) store_any(dw + (u64)block * size + at, sum(vec{}, at));
        return;
    }
    for (u64 i = at; i < at + V && i < stride; ++i) {
        if (i < size ? !dw : !db) continue;
        (i < size ? dw[(u64)block * size + i] : db[(u64)block * n + (i - size)]) = sum(0.0f, i);
    }
}

// Which kernel a product of rows takes, and whether the 8-bit form of a is written by itself, in front of it.
enum class RowsKernel { few, wide, narrow, all };
struct RowsChoice {
    RowsKernel kernel;
    bool pack;
};
RowsChoice rows_choice(const RowsArgs &r, u32 dtype)
{
    const bool wide = dtype == LMK_GS_BF16 && wide_rows_fit(r), narrow = dtype == LMK_GS_F32 && narrow_rows_fit(r);
    const bool few = few_rows_fit(r, wide) && !(narrow && r.keep_codes);
    return RowsChoice{few ? RowsKernel::few : wide ? RowsKernel::wide : narrow ? RowsKernel::narrow : RowsKernel::all,
                      r.keep_codes && (few || !(wide || narrow))};
}
// of its largest launch
u64 rows_threads(const RowsArgs &r, u32 dtype, bool across)
{
    const RowsChoice choice = rows_choice(r, dtype);
    const u64 pack = choice.pack ? checkpoint8_threads(r.rows, r.sums) : 0;
    const u64 product = choice.kernel == RowsKernel::few      ? few_rows_threads(r, across)
                        : choice.kernel == RowsKernel::wide   ? wide_rows_threads(r)
                        : choice.kernel == RowsKernel::narrow ? narrow_rows_threads(r)
                                                              : max_runs(r.rows, r.blocks, kTile) * ((r.cols + kTile - 1) / kTile) * kThreads;
    return pack > product ? pack : product;
}

template <class T, bool ACROSS>
hipError_t rows_go(RowsArgs r, u32 gate, hipStream_t stream)
{
    r.col_tiles = (r.cols + kTile - 1) / kTile;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kTile) * r.col_tiles);
    if (gate == 0) hipLaunchKernelGGL((rows_kernel<T, ACROSS, 0>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    else if (gate == 1) hipLaunchKernelGGL((rows_kernel<T, ACROSS, 1>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    else hipLaunchKernelGGL((rows_kernel<T, ACROSS, 2>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    return hipGetLastError();
}
template <class T>
hipError_t rows_as(RowsArgs r, bool across, hipStream_t stream)
{
    constexpr u32 dtype = std::is_same<T, float>::value ? LMK_GS_F32 : LMK_GS_BF16;
    const RowsChoice choice = rows_choice(r, dtype);
    if (choice.pack) {
        const lmk_gs_checkpoint8 keep = {reinterpret_cast<int8_t *>(r.keep_codes), r.keep_scale};
        const hipError_t e = launch_checkpoint8_pack(r.a, r.lda, r.rows, r.sums, dtype, r.offsets, r.blocks, keep, stream);
        if (e != hipSuccess) return e;
    }
    if (choice.kernel == RowsKernel::few) return launch_few_rows(r, dtype, across, stream);
    if (choice.kernel == RowsKernel::wide) return launch_wide_rows(r, across, stream);
    if (choice.kernel == RowsKernel::narrow) return launch_narrow_rows(r, across, stream);
    const u32 gate = !r.gate ? 0 : r.gate_scale ? 2 : 1;
    return across ? rows_go<T, true>(r, gate, stream) : rows_go<T, false>(r, gate, stream);
}

// kind: as sums_kernel's
bool sums_wide(const SumsArgs &r, u32 dtype, u32 kind) { return dtype == LMK_GS_BF16 && kind != 0 && wide_sums_fit(r); }
u64 sums_threads(const SumsArgs &r, u32 dtype, u32 kind)
{
    if (sums_wide(r, dtype, kind)) return wide_sums_threads(r);
    return (u64)r.slices * ((r.n + kTile - 1) / kTile) * (kind == 0 ? 1 : (r.k + kTile - 1) / kTile) * kThreads;
}

template <class T>
hipError_t sums_as(SumsArgs r, u32 kind, hipStream_t stream)
{
    if (sums_wide(r, std::is_same<T, float>::value ? LMK_GS_F32 : LMK_GS_BF16, kind)) return launch_wide_sums(r, stream);
    r.n_tiles = (r.n + kTile - 1) / kTile;
    r.k_tiles = kind == 0 ? 1 : (r.k + kTile - 1) / kTile;
    r.tiles = (u32)((u64)r.slices * r.n_tiles * r.k_tiles);
    if (kind == 2) hipLaunchKernelGGL((sums_kernel<T, 2>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    else if (kind == 1) hipLaunchKernelGGL((sums_kernel<T, 1>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    else hipLaunchKernelGGL((sums_kernel<T, 0>), dim3(r.tiles), dim3(kThreads), 0, stream, r);
    return hipGetLastError();
}

}  // namespace

// Small matrices in float32 take one pass over the rows for all three gradients; the rest of the rule (strides) is the
// arrays', and what does not fit takes the other kernels with the same slices.  At the limit the two are even (24 blocks of 96 x 64,
// one pass / the others: 300 000 rows 127 / 122 us, 20 000 rows 26.5 / 27.7; 80 x 64: 108 / 115, 23.4 / 25.8).
static bool one_pass(const lmk_gs_linear &l) { return l.dtype == LMK_GS_F32 && l.n <= 96 && l.k <= 64; }

// how the sums over rows are shared out
struct RunPlan {
    u32 per, slices;        // rows of a run or slice; sets of partial sums, less the blocks
    u32 side;               // of the bfloat16 kernel's tiles
};
static RunPlan run_plan(const lmk_gs_linear &l)
{
    const u64 sums = (u64)l.n * l.k + l.n;
    RunPlan p = {};
    if (one_pass(l)) {
        // a run's own costs (the weights into LDS, the sums out of registers) are those of some hundred rows: one run a workgroup,
        // all of them at once, whole tiles for each wavefront
        const u32 most = narrow_backward_slots(l.n, l.k), slots = most - (l.blocks < most / 2 ? l.blocks : most / 2);
        p.per = (u32)(((u64)l.rows + slots * 64 - 1) / (slots * 64)) * 64;
        p.per = p.per < 64 ? 64 : p.per;
        p.slices = l.rows / p.per + 1;
    } else {
        // time of a row of a tile: its products at the rate (flop a us) that a compute unit's share of the tiles reaches
        const auto look = [&](u32 side, u32 slots, double rate, double run_us) {
            const u64 pairs = (u64)((l.n + side - 1) / side) * ((l.k + side - 1) / side);
            return slices_of(l.rows, l.blocks, pairs, slots, 2.0 * side * side * slots / rate, run_us, sums);
        };
        if (l.dtype == LMK_GS_F32) {
            p.slices = look(kTile, 1024, 1e8, 6.0).count;
        } else {
            // large tiles read less, small ones have less of a run's own costs, two workgroups a compute unit (8 blocks of
            // 1024 x 1024, large / small: 4000 rows 57 / 42 us; 64 of 256 x 512, 1500 rows 60 / 32; 65 536 rows of 1024 x 1024
            // in large ones)
            const Slices small = look(128, 512, 0.8e9, 4.0), large = look(256, 256, 1e9, 10.0);
            p.side = large.us < small.us ? 256 : 128;
            p.slices = p.side == 256 ? large.count : small.count;
        }
        p.per = rows_of_slice(l.rows, p.slices);
    }
    return p;
}

// How the partial sums are joined
struct JoinShape {
    bool many, parts;
    u32 pieces;             // workgroups of a block
};
static JoinShape join_shape(const lmk_gs_linear &l, const RunPlan &plan)
{
    // few sums are many sets each, and latency; many are bytes (24 blocks of 96 x 35, 300 000 rows, gradients with
    // few as many and as few: 94 / 93 us; one block: 128 / 97; 4 blocks of 1024 x 1024, 1000 rows: 33 / 38)
    const u64 stride = (u64)l.n * l.k + l.n;
    JoinShape j;
    j.many = stride * l.blocks >= 1u << 20;
    // few sets a block are not worth parts (7 blocks of 131 x 257, 71 sets: 7.5 us with them, 4.0 without)
    j.parts = !j.many && plan.slices / l.blocks >= 16;
    const u32 width = j.many ? 1024 : j.parts ? 32 : 256;
    j.pieces = (u32)((stride + width - 1) / width);
    return j;
}

// ---- what the calls hand to the kernels
static RowsArgs forward_args(const lmk_gs_linear &l, const void *x, u64 ldx, const float *bias, bool relu, void *y, u64 ldy,
                             const lmk_gs_checkpoint8 *keep)
{
    RowsArgs r = {};
    if (keep) {
        r.keep_codes = reinterpret_cast<u32 *>(keep->codes);
        r.keep_scale = keep->scale;
    }
    r.a = x; r.lda = ldx;
    r.w = l.w; r.ldw = l.ldw; r.w_block = l.w_block;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.cols = l.n; r.sums = l.k;
    r.out = y; r.ldo = ldy; r.bias = bias; r.relu = relu;
    return r;
}
static RowsArgs dx_args(const lmk_gs_linear &l, const void *dy, u64 lddy, const void *x, u64 ldx, const lmk_gs_checkpoint8 *kept,
                        bool gate, const lmk_gs_linear_grads &out)
{
    RowsArgs r = {};
    r.a = dy; r.lda = lddy;
    r.w = l.w; r.ldw = l.ldw; r.w_block = l.w_block;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.cols = l.k; r.sums = l.n;
    r.out = out.dx; r.ldo = out.lddx;
    if (gate) {
        r.gate = kept ? (const void *)kept->codes : x;
        r.ldgate = kept ? (l.k + 31) / 32 * 32 : ldx;
        r.gate_scale = kept ? kept->scale : nullptr;
    }
    return r;
}
static SumsArgs sums_args(const lmk_gs_linear &l, const RunPlan &plan, const void *dy, u64 lddy, const void *x, u64 ldx,
                          const lmk_gs_checkpoint8 *kept, const lmk_gs_linear_grads &out, float *part)
{
    SumsArgs r = {};
    r.dy = dy; r.lddy = lddy;
    r.x = kept ? (const void *)kept->codes : x;
    r.ldx = ldx;
    r.scale = kept ? kept->scale : nullptr;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.n = l.n; r.k = l.k;
    r.dw = out.dw; r.db = out.db; r.in_major = l.in_major;
    r.part = part;
    r.slices = plan.slices;
    r.side = plan.side;
    r.per = plan.per;
    return r;
}
static u32 sums_kind(const lmk_gs_linear_grads &out, const lmk_gs_checkpoint8 *kept) { return !out.dw ? 0 : kept ? 2 : 1; }
static BackwardArgs one_pass_args(const lmk_gs_linear &l, const RunPlan &plan, const void *dy, u64 lddy, const void *x, u64 ldx,
                                  const lmk_gs_checkpoint8 *kept, bool gate, const lmk_gs_linear_grads &out, float *part)
{
    BackwardArgs r = {};
    r.dy = static_cast<const float *>(dy); r.lddy = lddy;
    if (out.dw || (out.dx && gate)) {
        r.x = kept ? (const void *)kept->codes : x;
        r.ldx = ldx;
        r.scale = kept ? kept->scale : nullptr;
    }
    r.w = static_cast<const float *>(l.w); r.ldw = l.ldw; r.w_block = l.w_block;
    r.offsets = l.offsets; r.blocks = l.blocks; r.rows = l.rows; r.n = l.n; r.k = l.k;
    r.in_major = l.in_major; r.gate = gate;
    r.dx = static_cast<float *>(out.dx); r.lddx = out.lddx; r.dw = out.dw; r.db = out.db;
    r.part = part; r.runs = plan.slices + l.blocks; r.per = plan.per;
    return r;
}

// ---- whether every launch of a call has fewer threads than a launch holds, asked before the first one
bool grouped_linear_fits(const lmk_gs_linear &l, const void *x, u64 ldx, void *y, u64 ldy, const lmk_gs_checkpoint8 *keep)
{
    return rows_threads(forward_args(l, x, ldx, nullptr, false, y, ldy, keep), l.dtype, l.in_major != 0) < kMostThreads;
}

bool grouped_backward_fits(const lmk_gs_linear &l, const void *dy, u64 lddy, const void *x, u64 ldx, const lmk_gs_checkpoint8 *kept,
                           bool gate, const lmk_gs_linear_grads &out)
{
    const bool sums = out.dw || out.db;
    const RunPlan plan = sums ? run_plan(l) : RunPlan{};
    if (sums && (u64)join_shape(l, plan).pieces * l.blocks * kThreads >= kMostThreads) return false;
    // one pass takes a workgroup a run, of which there are at most some 1000 and one a block
    if (sums && one_pass(l) && narrow_backward_fits(one_pass_args(l, plan, dy, lddy, x, ldx, kept, gate, out, nullptr), kept != nullptr)) return true;
    if (out.dx && rows_threads(dx_args(l, dy, lddy, x, ldx, kept, gate, out), l.dtype, l.in_major == 0) >= kMostThreads) return false;
    return !sums || sums_threads(sums_args(l, plan, dy, lddy, x, ldx, kept, out, nullptr), l.dtype, sums_kind(out, kept)) < kMostThreads;
}

size_t grouped_backward_bytes(const lmk_gs_linear &l)
{
    return (size_t)(((u64)run_plan(l).slices + l.blocks) * ((u64)l.n * l.k + l.n) * 4);
}

hipError_t launch_grouped_linear(const lmk_gs_linear &l, const void *x, u64 ldx, const float *bias, bool relu, void *y,
                                 u64 ldy, const lmk_gs_checkpoint8 *keep, hipStream_t stream)
{
    const RowsArgs r = forward_args(l, x, ldx, bias, relu, y, ldy, keep);
    return l.dtype == LMK_GS_F32 ? rows_as<float>(r, l.in_major != 0, stream) : rows_as<__bf16>(r, l.in_major != 0, stream);
}

hipError_t launch_grouped_backward(const lmk_gs_linear &l, const void *dy, u64 lddy, const void *x, u64 ldx,
                                   const lmk_gs_checkpoint8 *kept, bool gate, const lmk_gs_linear_grads &out,
                                   char *workspace, hipStream_t stream)
{
    const bool sums = out.dw || out.db;
    const RunPlan plan = sums ? run_plan(l) : RunPlan{};
    float *part = reinterpret_cast<float *>(workspace);
    const auto join = [&](bool by_blocks) {
        const JoinShape j = join_shape(l, plan);
        auto kernel = j.many ? join_kernel<4, 4, 1> : j.parts ? join_kernel<1, 4, 8> : join_kernel<1, 8, 1>;
        hipLaunchKernelGGL(kernel, dim3(j.pieces * l.blocks), dim3(kThreads), 0, stream, l.offsets, l.blocks, l.rows, plan.per, by_blocks, part,
                           l.n, l.k, out.dw, out.db, j.pieces);
        return hipGetLastError();
    };
    if (sums && one_pass(l)) {
        const BackwardArgs r = one_pass_args(l, plan, dy, lddy, x, ldx, kept, gate, out, part);
        if (narrow_backward_fits(r, kept != nullptr)) {
            const hipError_t e = launch_narrow_backward(r, kept != nullptr, stream);
            return e == hipSuccess ? join(true) : e;
        }
    }
    if (out.dx && l.rows > 0) {
        const RowsArgs r = dx_args(l, dy, lddy, x, ldx, kept, gate, out);
        const hipError_t e = l.dtype == LMK_GS_F32 ? rows_as<float>(r, l.in_major == 0, stream) : rows_as<__bf16>(r, l.in_major == 0, stream);
        if (e != hipSuccess) return e;
    }
    if (!sums) return hipSuccess;
    const SumsArgs r = sums_args(l, plan, dy, lddy, x, ldx, kept, out, part);
    const u32 kind = sums_kind(out, kept);
    const hipError_t e = l.dtype == LMK_GS_F32 ? sums_as<float>(r, kind, stream) : sums_as<__bf16>(r, kind, stream);
    return e == hipSuccess ? join(false) : e;
}

}  // namespace lmk
