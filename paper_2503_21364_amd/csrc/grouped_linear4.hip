// Layers whose weights belong to blocks of rows, both operands in 4 bits (lmk_gs_grouped_linear4): y = act(x w_g^T + b_g) on
// v_mfma_scale_f32_16x16x128_f8f6f4.  A lane feeds 32 codes, 16 bytes, of one row and their scale byte; the products of codes and powers of two are
// exact, sums are in 32 bits.
//
// 8192 x 8192 x 8192 258 us, 4.3 PFLOP/s; 65 536 rows of 2048 -> 2048 in 16 even blocks 171 us (3.2; 268 MB of results in bfloat16 alone take 52), in
// ragged ones, whose last tiles are partly empty, 186 of the same inputs again and again, 188 to 195 behind their packing, 207 of others, 213 behind a
// fill of 268 MB.  Bound by LDS and its loads: a step's fragments and scales take it as long as their products take the
// matrix instructions, which reach 7 PFLOP/s by themselves.
#include "block4.h"
#include "grouped_wide.h"

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
    bool past;                  // y is more than the caches of the dies hold
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
// 64 outputs where that fills the compute units (128 rows, one block of 2048 -> 2048, 64 / 16: 7.0 / 9.5 us; 24 rows, 64 blocks of 1024 -> 2048 8.2 /
// 11.3), 16 where not (one row, 8 blocks of 4096 -> 4096: 9.5 / 4.3)
u32 few_columns(const Linear4Args &r) { return max_runs(r.rows, r.blocks, kRows) * ((r.n + 63) / 64) >= 320 ? 64 : 16; }

// ---- tiles, as in grouped_wide.hip: a row's 256 codes are the 128 bytes that 64 bfloat16 are there, and come into LDS by the same loads, and a
// lane's fragment is the 16 bytes with one scale.  The scales of 512 values of a row are 16 bytes; they come every second pair of steps, 64
// rows a load, and a lane reads the four bytes of a step and takes its own.

// of P and Q together, rows of a tile
template <u32 TP, u32 TQ, u32 WAVES> struct Scales4 {
    static_assert((TP + TQ) / 64 == WAVES && TP % 64 == 0, "one load a wavefront");
    __amdgpu_buffer_rsrc_t from;        // this wavefront's rows: of P or of Q
    u32 at;                             // this lane's row
    u32 shift, p_read, q_read;

    __device__ __forceinline__ void init(const uint8_t *p, u32 p_rows, const uint8_t *q, u32 q_rows, u32 bytes, u32 wave, u32 lane, u32 p0, u32 q0)
    {
        const bool of_p = wave < TP / 64;
        from = buffer_of(reinterpret_cast<const void *>(uniform64(reinterpret_cast<u64>(of_p ? p : q))), uniform((of_p ? p_rows : q_rows) * bytes));
        at = ((of_p ? wave : wave - TP / 64) * 64 + lane) * bytes;
        shift = 8 * (lane >> 4);
        p_read = (p0 + (lane & 15)) * 16;
        q_read = (TP + q0 + (lane & 15)) * 16;
    }
    __device__ __forceinline__ void fill(lds_char *lds, u32 wave)
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds + wave * 1024, 16, (int)at, 0, 0, 0);
        at += 16;
    }
    __device__ __forceinline__ u32 of(const lds_char *lds, u32 read, u32 f, u32 step) const
    {
        return *reinterpret_cast<const __attribute__((address_space(3))) u32 *>(lds + read + f * 256 + step * 4) >> shift;
    }
};

// A workgroup takes tiles one after the other.  The next one's first loads are on their way before this one's results leave, and the stores,
// which take as long as several steps, are not waited for until the next tile's second pair has to be there (vector memory operations
// complete in order: what was asked for before the last kStores stores has arrived once no more than those are left).
template <class T, class S, u32 TP, u32 TQ, u32 WP>
__global__ __launch_bounds__(S::kThreads, 2) void wide_rows4_kernel(const Linear4Args r)
{
    extern __shared__ __align__(16) char wide_lds[];
    constexpr u32 kScales = (TP + TQ) * 16, kStores = S::kP * S::kQ / (sizeof(T) == 2 ? 2 : 1);
    const u32 lane = threadIdx.x & (kWave - 1), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 p0 = wave % WP * (S::kP * 16), q0 = wave / WP * (S::kQ * 16);
    const u32 row_bytes = code_bytes(r.k), scales = scale_bytes(r.k), steps = row_bytes / 64;
    lds_char *lds = (lds_char *)wide_lds, *lp = lds, *lq = lds + 2 * S::kPartP, *ls = lds + S::kLds, *lb = ls + 2 * kScales;

    // the tile: block ~0u for rows of no block
    struct Tile {
        u32 block, row0, height, col0, width;
    };
    // the next one from number `id` on that there is
    const auto locate = [&](u32 &id, Tile &to) {
        for (; id < r.tiles; id += gridDim.x) {
            const u32 tile = tile_of_workgroup(id, r.tiles, S::kResident * kUnits);
            // four rows of tiles beside each other: what a die works on at once is four by eight of them, and shares most of its operands
            const u32 band = tile / (4 * r.col_tiles), in = tile - band * 4 * r.col_tiles, row_tile = 4 * band + in % 4;
            const RowRun run = find_run(r.offsets, r.blocks, r.rows, TQ, row_tile);
            if (!run.found) continue;
            to.block = uniform(run.block);
            to.row0 = uniform(run.begin + run.local * TQ);
            to.height = uniform(run.end - to.row0 < TQ ? run.end - to.row0 : TQ);
            to.col0 = uniform(in / 4 * TP);
            to.width = uniform(r.n - to.col0 < TP ? r.n - to.col0 : TP);
            return true;
        }
        return false;
    };
    Along16<TP, S::kWaves> p;
    Along16<TQ, S::kWaves> q;
    Scales4<TP, TQ, S::kWaves> sc;
    // `part` of the codes; the scales of steps 4 i and on are in half i % 2 of theirs
    const auto fill = [&](u32 part, u32 pair) {
        p.fill(lp + part * S::kPartP, wave);
        q.fill(lq + part * S::kPartQ, wave);
        if (pair % 2 == 0) sc.fill(ls + (pair / 2 & 1) * kScales, wave);
    };
    const auto begin = [&](const Tile &t) {
        if (t.block == ~0u) return;
        const u32 at = afresh(lane);
        const u64 wrow = (u64)t.block * r.n + t.col0;
        const auto first_of = [](const char *of, u64 bytes) { return reinterpret_cast<const __bf16 *>(uniform64(reinterpret_cast<u64>(of) + bytes)); };
        p.init(first_of(r.w, wrow * row_bytes), row_bytes / 2, t.width, row_bytes / 2, wave, at);
        q.init(first_of(r.x, (u64)t.row0 * row_bytes), row_bytes / 2, t.height, row_bytes / 2, wave, at);
        sc.init(r.ws + wrow * scales, t.width, r.xs + (u64)t.row0 * scales, t.height, scales, wave, at, p0, q0);
        if (wave < TP / kWave) {
            const u64 bias = r.bias ? reinterpret_cast<u64>(r.bias + wrow) : reinterpret_cast<u64>(r.offsets);
            const __amdgpu_buffer_rsrc_t from = buffer_of(reinterpret_cast<const void *>(uniform64(bias)), r.bias ? uniform(t.width * 4) : 0u);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lb + wave * kWave * 4, 4, (int)((wave * kWave + at) * 4), 0, 0, 0);
        }
        fill(0, 0);
        fill(1, 1);
    };

    u32 id = blockIdx.x;
    Tile tile;
    if (!locate(id, tile)) return;
    wavefronts_meet<0x070>();               // nothing but those loads is on its way, here as for every other tile
    begin(tile);
    bool counted = false;
    for (;;) {
        if (counted) wavefronts_meet<(kStores & 15) | (kStores >> 4) << 14 | 0x070>();
        else wavefronts_meet<0x070>();
        // the sums begin with the bias
        f32x4 acc[S::kP][S::kQ];
        const lds_char *own_bias = lb + (p0 + 4 * (afresh(lane) >> 4)) * 4;
#pragma unroll
        for (u32 i = 0; i < S::kP; ++i) {
            const f32x4 b = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(own_bias + 64 * i);
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j) acc[i][j] = tile.block != ~0u ? b : f32x4{};
        }
        if (tile.block != ~0u) {
            i32x4 fp[S::kP], fq[2][S::kQ];
            u32 sp[S::kP], sq[2][S::kQ];
            // step t of eight, of which two pairs have the codes' parts and four the halves of the scales in turns
            auto read_p = [&](u32 i, u32 t) {
                fp[i] = __builtin_bit_cast(i32x4, p.fragment(lp + (t / 2 & 1) * S::kPartP, t & 1, p0, i));
                sp[i] = sc.of(ls + (t / 4 & 1) * kScales, sc.p_read, i, t & 3);
            };
            auto read_q = [&](u32 j, u32 t) {
                fq[t & 1][j] = __builtin_bit_cast(i32x4, q.fragment(lq + (t / 2 & 1) * S::kPartQ, t & 1, q0, j));
                sq[t & 1][j] = sc.of(ls + (t / 4 & 1) * kScales, sc.q_read, j, t & 3);
            };
            // multiplies step t and reads the fragments of the next: those of P take the place of what has been used
            auto step = [&](u32 t) {
#pragma unroll
                for (u32 j = 0; j < S::kQ; ++j) read_q(j, t + 1);
#pragma unroll
                for (u32 i = 0; i < S::kP; ++i) {
#pragma unroll
                    for (u32 j = 0; j < S::kQ; ++j) acc[i][j] = product4(fp[i], sp[i], fq[t & 1][j], sq[t & 1][j], acc[i][j]);
                    read_p(i, t + 1);
                }
                asm volatile("" ::: "memory");              // the reads stay in this step
            };
#pragma unroll
            for (u32 i = 0; i < S::kP; ++i) read_p(i, 0);
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j) read_q(j, 0);
            for (u32 t0 = 0; t0 < steps; t0 += 8) {
#pragma unroll
                for (u32 t = 0; t < 8; t += 2) {
                    if (t0 + t >= steps) break;
                    step(t);
                    if (t0 + t + 1 >= steps) break;
                    // the next pair has arrived, and this pair's fragments have left LDS
                    wavefronts_meet<0x070>();
                    fill(t / 2 & 1, t / 2 + 2);
                    step(t + 1);
                }
            }
        }
        const Tile done = tile;
        id += gridDim.x;
        const bool more = locate(id, tile);
        // nothing may be on its way into LDS when it is filled for the next tile, or when the workgroup ends
        wavefronts_meet<0x070>();
        if (more) begin(tile);
        asm volatile("" ::: "memory");                      // the stores stay behind those loads
        if (r.relu) {
#pragma unroll
            for (u32 i = 0; i < S::kP; ++i)
#pragma unroll
                for (u32 j = 0; j < S::kQ; ++j) acc[i][j] = __builtin_elementwise_maximum(acc[i][j], f32x4{});          // NaN stays
        }
        T *out = static_cast<T *>(r.y) + (u64)done.row0 * r.ldy + done.col0;
        // `all`: every result of the tile is there; `past`: past the caches
        const u32 at = afresh(lane), group = at >> 4;               // where its results go is not held through the product
        const auto store = [&](auto all, auto past) {
            if constexpr (all) stores_begin<kStores>();
#pragma unroll
            for (u32 j = 0; j < S::kQ; ++j) {
                if constexpr (sizeof(T) == 2) {
                    // Two neighbouring results exchange lanes: eight consecutive values a lane, 64 bytes a row; then two of those, lanes eight
                    // rows apart: whole lines, of rows row % 8 and of the next eight.
                    const auto eight = [&](u32 i) {
                        const u32x2 a = __builtin_amdgcn_permlane16_swap(pack_bf16(acc[i][j][0], acc[i][j][1]), pack_bf16(acc[i + 1][j][0], acc[i + 1][j][1]), false, false);
                        const u32x2 b = __builtin_amdgcn_permlane16_swap(pack_bf16(acc[i][j][2], acc[i][j][3]), pack_bf16(acc[i + 1][j][2], acc[i + 1][j][3]), false, false);
                        return u32x4{a[0], b[0], a[1], b[1]};
                    };
#pragma unroll
                    for (u32 i = 0; i < S::kP; i += 4) {
                        const u32x4 lo = eight(i), hi = eight(i + 2);
                        u32x4 v[2];
#pragma unroll
                        for (u32 e = 0; e < 4; ++e) {
                            v[0][e] = (u32)__builtin_amdgcn_update_dpp((int)lo[e], (int)hi[e], 0x128, 0xf, 0xc, false);         // row_ror:8
                            v[1][e] = (u32)__builtin_amdgcn_update_dpp((int)hi[e], (int)lo[e], 0x128, 0xf, 0x3, false);
                        }
                        const u32 c = p0 + 16 * (i + (group & 1)) + 8 * (group >> 1) + (at & 8) * 4;
#pragma unroll
                        for (u32 h = 0; h < 2; ++h) {
                            const u32 row = q0 + 16 * j + (at & 7) + 8 * h;
                            T *to = out + (u64)row * r.ldy;
                            if (all || (row < done.height && c + 8 <= done.width)) {
                                store_vector<past>(to + c, v[h]);
                            } else if (row < done.height) {
#pragma unroll
                                for (u32 e = 0; e < 7; ++e)
                                    if (c + e < done.width) to[c + e] = __builtin_bit_cast(__bf16, (unsigned short)(v[h][e / 2] >> (16 * (e % 2))));
                            }
                        }
                    }
                } else {
                    const u32 row = q0 + 16 * j + (at & 15);
                    T *to = out + (u64)row * r.ldy;
#pragma unroll
                    for (u32 i = 0; i < S::kP; ++i) {
                        const u32 c = p0 + 16 * i + 4 * group;
                        if (all || (row < done.height && c + 4 <= done.width)) {
                            store_vector<past>(to + c, acc[i][j]);
                        } else if (row < done.height) {
#pragma unroll
                            for (u32 v = 0; v < 3; ++v)
                                if (c + v < done.width) to[c + v] = acc[i][j][v];
                        }
                    }
                }
            }
            if constexpr (all) stores_end();
        };
        counted = done.height == TQ && done.width == TP;
        if (sizeof(T) == 2 && counted && r.past) store(std::true_type{}, std::bool_constant<sizeof(T) == 2>{});
        else if (counted) store(std::true_type{}, std::false_type{});
        else store(std::false_type{}, std::false_type{});
        if (!more) return;
    }
}

template <class T, u32 TP, u32 TQ, u32 WP, u32 WQ> hipError_t wide_go(Linear4Args r, hipStream_t stream)
{
    using S = Shape<TP, TQ, WP, WQ>;
    constexpr u32 lds = S::kLds + 2 * (TP + TQ) * 16 + TP * 4;
    // 64 bytes of a row a store in float32, half a line: through the caches (30 000 rows of 512 -> 1024: 40 us, so 31)
    r.past = sizeof(T) == 2 && past_caches(r.y, r.ldy * sizeof(T), (u64)r.rows * r.n * sizeof(T));
    r.col_tiles = (r.n + TP - 1) / TP;
    r.tiles = (u32)((max_runs(r.rows, r.blocks, TQ) + 3) / 4 * 4 * r.col_tiles);
    auto kernel = wide_rows4_kernel<T, S, TP, TQ, WP>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    const u32 at_once = 8 * kUnits * S::kResident;
    hipLaunchKernelGGL(kernel, dim3(r.tiles < at_once ? r.tiles : at_once), dim3(S::kThreads), lds, stream, r);
    return hipGetLastError();
}
// As in grouped_wide.hip.  256 x 256 / 128 x 128, 8 blocks of 1024 -> 1024: 4096 rows 15.6 / 10.2 us, 16 384 18.9 / 21.3, 65 536 61 / 72;
// 10 007 rows in 7 of 1000 -> 257 18.3 / 11.1; 8192 x 8192 x 8192 262 / 321.
bool large_tiles(const Linear4Args &r)
{
    const auto share = [&](u32 side) { return __builtin_ceilf((float)r.rows / side + 0.5f * (r.blocks - 1)) * ((r.n + side - 1) / side); };
    return __builtin_ceilf(share(256) / 256) < 0.7f * share(128) / 512;
}
// This kernel / tiles: one row, 8 blocks of 4096 -> 4096 4.3 / 12.9 us; 128 rows, one block of 2048 -> 2048 7.1 / 8.7, 8 of 1024 -> 1024 4.2 / 6.0;
// 64 blocks of 1024 -> 2048, 24 rows 8.1 / 7.6
bool few_fit(const Linear4Args &r)
{
    const u64 row_tiles = r.rows < r.blocks ? r.rows : r.blocks;
    return (r.rows <= 128 || r.rows / 16 <= r.blocks) && row_tiles * ((r.n + 127) / 128) < 512;
}

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
    if (few_fit(r)) return few_columns(r) == 64 ? few_go<T, 64>(r, stream) : few_go<T, 16>(r, stream);
    return large_tiles(r) ? wide_go<T, 256, 256, 2, 4>(r, stream) : wide_go<T, 128, 128, 2, 2>(r, stream);
}

}  // namespace

bool grouped_linear4_fits(const lmk_gs_linear4 &l)
{
    const Linear4Args r = linear4_args(l, {}, nullptr, false, nullptr, 0);
    const u32 nt = few_fit(r) ? few_columns(r) : large_tiles(r) ? 256 : 128, per = few_fit(r) ? kRows : nt;
    return (max_runs(r.rows, r.blocks, per) + 3) * ((r.n + nt - 1) / nt) * (few_fit(r) ? 512 : 2 * nt) < kMostThreads;
}

hipError_t launch_grouped_linear4(const lmk_gs_linear4 &l, const lmk_gs_block4 &x, const float *bias, bool relu, void *y, u64 ldy,
                                  hipStream_t stream)
{
    const Linear4Args r = linear4_args(l, x, bias, relu, y, ldy);
    return l.dtype == LMK_GS_F32 ? linear4_as<float>(r, stream) : linear4_as<__bf16>(r, stream);
}

}  // namespace lmk
