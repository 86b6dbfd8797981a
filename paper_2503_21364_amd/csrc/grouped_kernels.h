// Arguments of the grouped layers' kernels, and what their launches share.
#ifndef LMK_GS_GROUPED_KERNELS_H
#define LMK_GS_GROUPED_KERNELS_H
#include "grouped.h"

#include <type_traits>

namespace lmk {

// rows of a block against its weights
struct RowsArgs {
    const void *a;              // [rows][sums]
    u64 lda;
    const void *w;              // block g at g * w_block
    u64 ldw, w_block;
    const u32 *offsets;
    u32 blocks, rows, cols, sums;
    void *out;                  // [rows][cols]
    u64 ldo;
    const float *bias;          // [blocks][cols] or NULL
    u32 relu;
    const void *gate;           // NULL, or what the result is gated with: values or codes
    u64 ldgate;                 // elements (codes) between its rows
    const uint8_t *gate_scale;  // of codes
    u32 tiles, col_tiles;
    u32 per;                    // rows of a run, where that is not fixed
    bool across;                // weights: columns contiguous, not sum indices
    u32 *keep_codes;            // NULL, or where the 8-bit form of a goes (small matrices and bfloat16 write it on the way)
    uint8_t *keep_scale;
};

// sums over the rows of a block
struct SumsArgs {
    const void *dy;             // [rows][n]
    u64 lddy;
    const void *x;              // [rows][k], or codes [rows][kp]
    u64 ldx;
    const uint8_t *scale;       // of codes
    const u32 *offsets;
    u32 blocks, rows, n, k;
    float *dw, *db;             // results, either may be NULL
    bool dw16;                  // dw is in bfloat16
    u32 in_major;
    float *part;                // partial sums: n k of dw, then n of db each
    u32 slices, per;            // of the rows, and rows of each
    u32 side;                   // of the bfloat16 kernel's tiles
    u32 tiles, n_tiles, k_tiles;
};

// all gradients of a layer of small matrices, float32
struct BackwardArgs {
    const float *dy;            // [rows][n]
    u64 lddy;
    const void *x;              // [rows][k] values, or codes [rows][kp]; NULL if neither dw nor the gate needs it
    u64 ldx;
    const uint8_t *scale;       // of codes
    const float *w;
    u64 ldw, w_block;
    const u32 *offsets;
    u32 blocks, rows, n, k;
    u32 in_major, gate;
    float *dx;                  // any of the three may be NULL
    u64 lddx;
    float *dw, *db;
    float *part;                // as SumsArgs
    u32 runs, per;              // sets of partial sums, rows of a run
    u32 shared;                 // floats of LDS of the weights
};

constexpr u32 kUnits = 32;        // compute units of a die

// Workgroups go to the eight dies in turn; this gives each die as many consecutive tiles as it runs at once, which share operands.
// One run of total / 8 tiles a die is slower: what the dies read then lies far apart (8192 x 8192 x 8192 in bfloat16, dx: 1022 us, so 873),
// and the last die has no work where `total` counts ends of blocks that there are not (16 384 rows x 512 x 512: 20 us, so 14).
__device__ __forceinline__ u32 tile_of_workgroup(u32 id, u32 total, u32 at_once)
{
    constexpr u32 dies = 8;
    const u32 round = dies * at_once, whole = total / round * round;
    const u32 i = id < whole ? id : id - whole, run = id < whole ? at_once : (total - whole) / dies;
    if (i >= run * dies && id >= whole) return id;
    const u32 die = i % dies, k = i / dies;
    return id < whole ? (k / run * dies + die) * run + k % run : whole + die * run + k;
}

// V consecutive values as they are in memory, so that a load on its way holds no more registers than it fills
template <class T, u32 V> using Run = T __attribute__((ext_vector_type(V)));

// How rows end: with whole runs of V values; anywhere, with a run at least in front of it; or before their first run does
enum class Ends { whole, any, early };
constexpr Ends ends_of(u32 count, u32 v) { return count % v == 0 ? Ends::whole : count >= v ? Ends::any : Ends::early; }

// V values of a row from `s` on; beyond `sums` zeros, but for rows that end anywhere, whose last V values they are there: a choice between the
// vector and single values would be waited for before the next load (408 rows of 76 blocks of 15 -> 1715 in float32 18.6 us, without it 10.6).  in_place moves them
// where they belong when they are used.
template <class T, u32 V, Ends ENDS> __device__ __forceinline__ Run<T, V> load_run(const T *p, u32 s, u32 sums)
{
    Run<T, V> v = {};
    if constexpr (ENDS == Ends::whole) {
        if (s < sums) v = load_any<Run<T, V>>(p + s);
    } else if constexpr (ENDS == Ends::any) {
        v = load_any<Run<T, V>>(p + (s + V <= sums ? s : sums - V));
    } else {
#pragma unroll
        for (u32 e = 0; e < V; ++e)
            if (s + e < sums) v[e] = p[s + e];
    }
    return v;
}
template <class T, u32 V> __device__ __forceinline__ void in_place(Run<T, V> &v, u32 s, u32 sums)
{
    v = moved(v, s + V <= sums ? 0u : s - (sums - V));
}

// `..._threads`: those that a launch would have
// Partial sums of blocks cut into runs of `per` rows (run r of block g is set r + g + (first row of g) / per): n k sums of dw and n of db a
// set; `slices`: sets, less the blocks.  Blocks of one run are not touched, those without rows get zeros.
u64 join_threads(u32 n, u32 k, u32 blocks, u32 slices);
hipError_t launch_join(const u32 *offsets, u32 blocks, u32 rows, u32 per, const float *part, u32 n, u32 k, float *dw, float *db, u32 slices,
                       hipStream_t stream);

// few rows, any type and alignment
bool few_rows_fit(const RowsArgs &r, bool wide);
u64 few_rows_threads(const RowsArgs &r, bool across);
hipError_t launch_few_rows(const RowsArgs &r, u32 dtype, bool across, hipStream_t stream);

// small matrices, float32
bool narrow_rows_fit(const RowsArgs &r);
u64 narrow_rows_threads(const RowsArgs &r);
hipError_t launch_narrow_rows(RowsArgs r, bool across, hipStream_t stream);

bool narrow_backward_fits(const BackwardArgs &r, bool codes);
u32 narrow_backward_slots(u32 n, u32 k);      // workgroups at once
hipError_t launch_narrow_backward(const BackwardArgs &r, bool codes, hipStream_t stream);

// bfloat16
bool wide_rows_fit(const RowsArgs &r);
u64 wide_rows_threads(const RowsArgs &r);
hipError_t launch_wide_rows(const RowsArgs &r, bool across, hipStream_t stream);
bool wide_sums_fit(const SumsArgs &r);
u64 wide_sums_threads(const SumsArgs &r);
hipError_t launch_wide_sums(const SumsArgs &r, hipStream_t stream);

}  // namespace lmk
#endif
