// Gated layers over few rows: as in grouped_few.hip a workgroup takes 16 rows and NT outputs, its eight wavefronts share out the sum
// indices and stream their part of both projections' weights straight into registers; the parts meet in LDS, where the activation and
// the product, or their gradients, are taken.
//
// Bound by the weights' bytes, and by a chain of latencies where they are few: one row of 8 blocks of 1024 -> 2048 in bfloat16 6.3 us; 128 rows of 8
// blocks of 1024 -> 1024 11 (33 MB, 3.0 TB/s); 512 rows of one in float32 46, where products take most of it (47 TFLOP/s).
#include "grouped_gated.h"

namespace lmk {

namespace {

constexpr u32 kRows = kGatedFewRows;

// BACKWARD: the gradients of both projections instead of y
template <class T, u32 NT, bool ACROSS, Ends ENDS, bool BACKWARD>
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
    const u32 lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), j = lane & 15, q = lane >> 4;
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
        Run<T, kC> across[kAhead][2][V];                // or kC columns of a sum index: the last ones of the row where fewer are left
        const u32 own = kC * j < width ? kC * j : 0u, left = r.n - col0;
        const int col = ENDS == Ends::any && own + kC > left ? (int)left - (int)kC : (int)own;
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V;
                const bool on = t0 + a < last;
                if (ENDS == Ends::any && !on) break;            // the same in all lanes
                const u32 sums = on ? r.k : 0u;
                fx[a] = load_run<T, V, ENDS>(x, s, sums);
#pragma unroll
                for (u32 h = 0; h < 2; ++h) {
                    if constexpr (ACROSS && ENDS == Ends::any) {
#pragma unroll
                        for (u32 e = 0; e < V; ++e)
                            across[a][h][e] = load_any<Run<T, kC>>(w + (u64)(s + e < sums ? s + e : sums - 1) * r.ldw + h * r.n + col0 + col);
                    } else if constexpr (ACROSS) {
#pragma unroll
                        for (u32 e = 0; e < V; ++e)
                            across[a][h][e] = load_run<T, kC, ENDS>(w + (u64)(s + e) * r.ldw + h * r.n + col0, kC * j, s + e < sums ? width : 0u);
                    } else {
#pragma unroll
                        for (u32 c = 0; c < kC; ++c) {
                            const u32 n = 16 * c + j;
                            along[a][h][c] = load_run<T, V, ENDS>(w + (u64)(h * r.n + col0 + (n < width ? n : 0)) * r.ldw, s, sums);
                        }
                    }
                }
            }
            if (ENDS == Ends::any && (t0 + kAhead > last || (t0 + kAhead) * step > r.k)) {
#pragma unroll
                for (u32 a = 0; a < kAhead; ++a) {
                    const u32 s = t0 + a < last ? (t0 + a) * step + q * V : r.k;
                    in_place<T, V>(fx[a], s, r.k);
#pragma unroll
                    for (u32 h = 0; h < 2; ++h) {
#pragma unroll
                        for (u32 c = 0; c < kC; ++c)
                            if constexpr (!ACROSS) in_place<T, V>(along[a][h][c], s, r.k);
#pragma unroll
                        for (u32 e = 0; e < V; ++e)
                            if (ACROSS && s + e >= r.k) across[a][h][e] = Run<T, kC>{};
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
                for (u32 v = 0; v < 4; ++v) {
                    // columns in front of the tile are another one's
                    const int at = !ACROSS ? (int)(16 * c + j) : ENDS == Ends::any ? col + (int)c : (int)(kC * j + c);
                    if (!ACROSS || ENDS != Ends::any || (at >= 0 && kC * j < width)) part[wave][4 * q + v][h * NT + at] = acc[h][c][v];
                }
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
            if (r.out32) {
                float *grads = static_cast<float *>(r.out) + (u64)(row0 + row) * r.ldo + col0 + c;
                grads[0] = da;
                grads[r.n] = du;
            } else {
                out[0] = (T)da;
                out[r.n] = (T)du;
            }
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

template <class T, u32 NT, bool ACROSS, Ends ENDS>
hipError_t few_go(GatedArgs r, hipStream_t stream)
{
    r.col_tiles = (r.n + NT - 1) / NT;
    r.tiles = (u32)(max_runs(r.rows, r.blocks, kRows) * r.col_tiles);
    if (r.dy) hipLaunchKernelGGL((gated_few_kernel<T, NT, ACROSS, ENDS, true>), dim3(r.tiles), dim3(512), 0, stream, r);
    else hipLaunchKernelGGL((gated_few_kernel<T, NT, ACROSS, ENDS, false>), dim3(r.tiles), dim3(512), 0, stream, r);
    return hipGetLastError();
}
// Outputs of a workgroup: 32 where that fills the compute units (512 rows, one block of 1024 -> 1024 in float32, 32 / 16 outputs: 46 / 54 us), 16
// where not (one row, 8 blocks of 1024 -> 2048 in bfloat16: 9.2 / 6.3)
u32 few_columns(const GatedArgs &r)
{
    return max_runs(r.rows, r.blocks, kRows) * ((r.n + 31) / 32) >= 320 ? 32 : 16;
}
template <class T, bool ACROSS>
hipError_t few_width(const GatedArgs &r, hipStream_t stream)
{
    constexpr u32 v = ACROSS ? 4 : 16 / sizeof(T);          // a run of x, and of the weights
    const bool wide = few_columns(r) == 32;
    const Ends sums = ends_of(r.k, v), cols = ACROSS && wide ? ends_of(r.n, 2) : Ends::whole;
    const bool single = sizeof(T) == 4 && !ACROSS && sums == Ends::any && r.k < 48;         // as in grouped_few.hip
    if (single || sums == Ends::early || cols == Ends::early)
        return wide ? few_go<T, 32, ACROSS, Ends::early>(r, stream) : few_go<T, 16, ACROSS, Ends::early>(r, stream);
    if (sums == Ends::any || cols == Ends::any) return wide ? few_go<T, 32, ACROSS, Ends::any>(r, stream) : few_go<T, 16, ACROSS, Ends::any>(r, stream);
    return wide ? few_go<T, 32, ACROSS, Ends::whole>(r, stream) : few_go<T, 16, ACROSS, Ends::whole>(r, stream);
}

// ---- dx, dW and db of few rows from the gradients of both projections in 32 bits, [rows][2 n]: one launch, since what a launch costs is more than
// its work here.  The first workgroups take dx, as above; the others 256 x 32 elements of one block's dW each, zeros where the block has no rows.
//
// FOUR: there are four sum indices and inputs or more.  Every load is then of four: the last ones begin four in front of the end, and what was
// there twice is either left out of the sum or stored twice, the same.

constexpr u32 kSumsP = 256, kSumsQ = 32;

struct FewGrads {
    const float *grads;
    u64 ldg;
    const void *x;
    u64 ldx;
    const void *w;
    u64 ldw, w_block;
    const u32 *offsets;
    u32 blocks, rows, n2, k;        // n2: outputs of both projections
    void *dx;
    u64 lddx;
    void *dw;
    float *db;
    u32 dx_groups, dx_cols;         // workgroups of dx, and of its columns
    u32 p_tiles, q_tiles;           // of a block's dW along its contiguous axis and across it
};

template <bool FOUR> __device__ __forceinline__ u32 four_from(u32 i, u32 count) { return FOUR && i + 4 > count ? count - 4 : i; }
template <bool FOUR, class T> __device__ __forceinline__ Run<T, 4> load_four(const T *p, u32 i, u32 count)
{
    return FOUR ? load_any<Run<T, 4>>(p + i) : load_run<T, 4, Ends::early>(p, i, count);
}

template <class T, u32 NT, bool IN_MAJOR, bool FOUR>
__device__ __forceinline__ void few_dx(const FewGrads &r, float (&part)[8][kRows][NT + 1])
{
    constexpr u32 kWaves = 8, kC = NT / 16, V = 4, kAhead = NT == 16 ? 8 : sizeof(T) == 4 ? 2 : 4;
    const u32 row_tile = blockIdx.x / r.dx_cols, col0 = (blockIdx.x - row_tile * r.dx_cols) * NT;
    const RowRun run = find_run(r.offsets, r.blocks, r.rows, kRows, row_tile);
    if (!run.found) return;
    const u32 row0 = run.begin + run.local * kRows;
    const u32 height = run.end - row0 < kRows ? run.end - row0 : kRows;
    const u32 width = r.k - col0 < NT ? r.k - col0 : NT;
    const u32 lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, j = lane & 15, q = lane >> 4;
    const bool inside = run.block != ~0u;
    if (inside) {
        f32x4 acc[kC] = {};
        const float *from = r.grads + (u64)(row0 + (j < height ? j : 0)) * r.ldg;
        const T *w = static_cast<const T *>(r.w) + (u64)run.block * r.w_block;
        // the lane's columns where they are contiguous, those behind the last one begin with the first of the tile
        const u32 own = kC * j < width ? col0 + kC * j : col0, col = kC == 4 ? four_from<FOUR>(own, r.k) : own;
        constexpr u32 step = 4 * V;
        const u32 all = (r.n2 + step - 1) / step, per = (all + kWaves - 1) / kWaves;
        const u32 first = wave * per, last = first + per < all ? first + per : all;
        Run<float, V> f[kAhead];
        Run<T, V> along[kAhead][kC];
        Run<T, kC> across[kAhead][V];
        for (u32 t0 = first; t0 < last; t0 += kAhead) {
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V, at = four_from<FOUR>(s, r.n2);
                f[a] = load_four<FOUR>(from, at, r.n2);
                if constexpr (IN_MAJOR) {
#pragma unroll
                    for (u32 c = 0; c < kC; ++c) {
                        const u32 m = 16 * c + j;
                        along[a][c] = load_four<FOUR>(w + (u64)(col0 + (m < width ? m : 0)) * r.ldw, at, r.n2);
                    }
                } else {
#pragma unroll
                    for (u32 e = 0; e < V; ++e) {
                        const u32 o = at + e < r.n2 ? at + e : r.n2 - 1;
                        if constexpr (FOUR) across[a][e] = load_any<Run<T, kC>>(w + (u64)o * r.ldw + col);
                        else across[a][e] = load_run<T, kC, Ends::early>(w + (u64)o * r.ldw, col, r.k);
                    }
                }
            }
#pragma unroll
            for (u32 a = 0; a < kAhead; ++a) {
                const u32 s = (t0 + a) * step + q * V, at = four_from<FOUR>(s, r.n2);
#pragma unroll
                for (u32 e = 0; e < V; ++e) {
                    // each sum index once, and neither factor of the others, which may not be finite
                    const bool on = t0 + a < last && at + e >= s && at + e < r.n2;
                    const float g = on ? f[a][e] : 0.0f;
#pragma unroll
                    for (u32 c = 0; c < kC; ++c)
                        acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(g, on ? to_f32(IN_MAJOR ? along[a][c][e] : across[a][e][c]) : 0.0f, acc[c], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (u32 c = 0; c < kC; ++c)
#pragma unroll
            for (u32 v = 0; v < 4; ++v) {
                // columns in front of the tile are another one's
                const int at = IN_MAJOR ? (int)(16 * c + j) : (int)(col + c) - (int)col0;
                if (at >= 0 && (IN_MAJOR || kC * j < width)) part[wave][4 * q + v][at] = acc[c][v];
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
        }
        static_cast<T *>(r.dx)[(u64)(row0 + row) * r.lddx + col0 + c] = (T)y;
    }
}

// A lane has four elements along the contiguous axis (P) and its wavefront four across it (Q); four rows of the block are on their way
// while four are multiplied.
template <class T, bool IN_MAJOR, bool FOUR> __device__ __forceinline__ void few_sums(const FewGrads &r)
{
    constexpr u32 kAhead = 4;
    using TP = typename std::conditional<IN_MAJOR, float, T>::type;
    using TQ = typename std::conditional<IN_MAJOR, T, float>::type;
    const u32 t = blockIdx.x - r.dx_groups, tiles = r.p_tiles * r.q_tiles, block = t / tiles, in = t - block * tiles;
    const u32 q_tile = in / r.p_tiles, p_tile = in - q_tile * r.p_tiles;
    const u32 lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
    const u32 pn = IN_MAJOR ? r.n2 : r.k, qn = IN_MAJOR ? r.k : r.n2;
    if (p_tile * kSumsP + 4 * lane >= pn || q_tile * kSumsQ + 4 * wave >= qn) return;           // nothing is waited for here
    const u32 p = four_from<FOUR>(p_tile * kSumsP + 4 * lane, pn), q = four_from<FOUR>(q_tile * kSumsQ + 4 * wave, qn);
    RowSlices all;
    all.init(r.offsets, r.blocks, r.rows, 1);
    u32 begin, end;
    all.block(block, begin, end);
    begin = uniform(begin);
    end = uniform(end);
    const TP *from_p = IN_MAJOR ? (const TP *)r.grads : (const TP *)r.x;
    const TQ *from_q = IN_MAJOR ? (const TQ *)r.x : (const TQ *)r.grads;
    const u64 ldp = IN_MAJOR ? r.ldg : r.ldx, ldq = IN_MAJOR ? r.ldx : r.ldg;
    f32x4 acc[4] = {}, sum = {};
    Run<TP, 4> vp[2][kAhead];
    Run<TQ, 4> vq[2][kAhead];
    const auto load = [&](u32 part, u32 row) {
#pragma unroll
        for (u32 i = 0; i < kAhead; ++i) {
            const u32 at = row + i < end ? row + i : begin;
            vp[part][i] = load_four<FOUR>(from_p + (u64)at * ldp, p, pn);
            vq[part][i] = load_four<FOUR>(from_q + (u64)at * ldq, q, qn);
        }
    };
    if (begin < end) load(0, begin);
    for (u32 row0 = begin; row0 < end; row0 += 2 * kAhead) {
#pragma unroll
        for (u32 part = 0; part < 2; ++part) {
            const u32 row = row0 + part * kAhead;
            if (row >= end) break;
            if (row + kAhead < end) load(1 - part, row + kAhead);
#pragma unroll
            for (u32 i = 0; i < kAhead; ++i) {
                if (row + i >= end) break;
                const f32x4 fp = {to_f32(vp[part][i][0]), to_f32(vp[part][i][1]), to_f32(vp[part][i][2]), to_f32(vp[part][i][3])};
                const f32x4 fq = {to_f32(vq[part][i][0]), to_f32(vq[part][i][1]), to_f32(vq[part][i][2]), to_f32(vq[part][i][3])};
#pragma unroll
                for (u32 c = 0; c < 4; ++c) acc[c] += fp * fq[c];
                sum += IN_MAJOR ? fp : fq;
            }
        }
    }
    if (r.dw) {
        T *dw = static_cast<T *>(r.dw) + (u64)block * qn * pn + (u64)q * pn + p;
#pragma unroll
        for (u32 c = 0; c < 4; ++c) {
            if constexpr (FOUR) {
                store4(dw + (u64)c * pn, acc[c]);
            } else if (q + c < qn) {
#pragma unroll
                for (u32 e = 0; e < 4; ++e)
                    if (p + e < pn) dw[(u64)c * pn + e] = (T)acc[c][e];
            }
        }
    }
    const u32 o = IN_MAJOR ? p : q;
    if (!r.db || (IN_MAJOR ? q_tile + wave : p_tile + lane) != 0) return;
#pragma unroll
    for (u32 e = 0; e < 4; ++e)
        if (FOUR || o + e < r.n2) r.db[(u64)block * r.n2 + o + e] = sum[e];
}

template <class T, u32 NT, bool IN_MAJOR, bool FOUR>
__global__ __launch_bounds__(512, 4) void gated_few_grads_kernel(const FewGrads r)
{
    __shared__ float part[8][kRows][NT + 1];
    if (blockIdx.x < r.dx_groups) few_dx<T, NT, IN_MAJOR, FOUR>(r, part);
    else few_sums<T, IN_MAJOR, FOUR>(r);
}

// Columns of dx of a workgroup, as in grouped_few.hip
u32 few_dx_columns(u32 rows, u32 blocks, u32 k, bool in_major)
{
    return max_runs(rows, blocks, kRows) * ((k + 63) / 64) >= (in_major ? 320 : 64) ? 64 : 16;
}

template <class T, bool IN_MAJOR> hipError_t few_grads_go(const FewGrads &r, u32 nt, hipStream_t stream)
{
    const u64 groups = r.dx_groups + (r.dw || r.db ? (u64)r.blocks * r.p_tiles * r.q_tiles : 0);
    const bool four = r.n2 >= 4 && r.k >= 4;
    const dim3 grid((u32)groups);
    if (groups == 0) return hipSuccess;
    if (nt == 64 && four) hipLaunchKernelGGL((gated_few_grads_kernel<T, 64, IN_MAJOR, true>), grid, dim3(512), 0, stream, r);
    else if (nt == 64) hipLaunchKernelGGL((gated_few_grads_kernel<T, 64, IN_MAJOR, false>), grid, dim3(512), 0, stream, r);
    else if (four) hipLaunchKernelGGL((gated_few_grads_kernel<T, 16, IN_MAJOR, true>), grid, dim3(512), 0, stream, r);
    else hipLaunchKernelGGL((gated_few_grads_kernel<T, 16, IN_MAJOR, false>), grid, dim3(512), 0, stream, r);
    return hipGetLastError();
}

}  // namespace

// As few_rows_fit.  This kernel / tiles: one row, 8 blocks of 1024 -> 2048 in bfloat16 6.3 / 9.7 us; 128 rows, 8 blocks of 1024 -> 1024 11.1 / 14.5,
// of one block 10.9 / 9.7; 64 blocks of 1024 -> 2048, 24 rows, where a tile a block fills the device, 48 both.  Float32: one block of 1024 -> 1024, 512
// rows 46 / 59; 8 of 512 -> 512, 1024 rows 25 / 32.
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

// Told from sizes alone.  Against the kernel above with the grouped layer's gradients, all of them: 26 blocks of 598 -> 431 in bfloat16, 56 rows
// 35 us / 84; 34 blocks of 156 -> 126, 16 rows 13 / 21; 64 blocks of 256 -> 256, 1024 rows 26 / 37; but 250 blocks of 256 -> 256 in float32, 4000
// rows 135 / 132, and one block of 1024 -> 1024, 128 rows 48 / 39: a block's rows are summed one after the other, which is also why they are
// not many in all, since they may be one block's (1000 rows in one of 64 blocks of 256 -> 256: 151 / 44).
bool gated_few_backward_fits(u32 rows, u32 blocks, u32 n, u32 k, u32 dtype)
{
    const u64 row_tiles = max_runs(rows, blocks, kRows), some = rows < blocks ? rows : blocks;
    const u64 sums = (u64)blocks * ((2 * n + kSumsQ - 1) / kSumsQ) * ((k + kSumsQ - 1) / kSumsQ);       // at least
    if ((row_tiles * ((n + 15) / 16) + row_tiles * ((k + 15) / 16) + sums) * 512 >= kMostThreads) return false;
    if (rows > 64 && (rows / 16 > blocks || rows > 512)) return false;
    return dtype == LMK_GS_F32 || (some * ((n + 63) / 64) < 512 && some * ((k + 127) / 128) < 512);
}

hipError_t launch_gated_few_backward(GatedArgs r, u32 dtype, float *grads, u64 ldg, void *dx, u64 lddx, void *dw, float *db, hipStream_t stream)
{
    r.out = grads;
    r.ldo = ldg;
    r.out32 = true;
    r.part = nullptr;
    if (r.rows > 0) {
        const hipError_t e = launch_gated_few(r, dtype, stream);
        if (e != hipSuccess) return e;
    }
    FewGrads f = {};
    f.grads = grads; f.ldg = ldg;
    f.x = r.x; f.ldx = r.ldx;
    f.w = r.w; f.ldw = r.ldw; f.w_block = r.w_block;
    f.offsets = r.offsets; f.blocks = r.blocks; f.rows = r.rows; f.n2 = 2 * r.n; f.k = r.k;
    f.dx = dx; f.lddx = lddx; f.dw = dw; f.db = db;
    const u32 nt = few_dx_columns(r.rows, r.blocks, r.k, r.in_major);
    f.dx_cols = (r.k + nt - 1) / nt;
    f.dx_groups = dx ? (u32)max_runs(r.rows, r.blocks, kRows) * f.dx_cols : 0u;
    const u32 pn = r.in_major ? f.n2 : f.k, qn = r.in_major ? f.k : f.n2;
    f.p_tiles = (pn + kSumsP - 1) / kSumsP;
    f.q_tiles = (qn + kSumsQ - 1) / kSumsQ;
    // the bias' gradient alone: the tiles of the first inputs
    if (!dw) (r.in_major ? f.q_tiles : f.p_tiles) = 1;
    if (dtype == LMK_GS_F32) return r.in_major ? few_grads_go<float, true>(f, nt, stream) : few_grads_go<float, false>(f, nt, stream);
    return r.in_major ? few_grads_go<__bf16, true>(f, nt, stream) : few_grads_go<__bf16, false>(f, nt, stream);
}

}  // namespace lmk
