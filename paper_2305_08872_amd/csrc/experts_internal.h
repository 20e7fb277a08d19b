// Declarations shared by the translation units of a mixture-of-experts layer's operators: the router, the products by
// groups of rows, the fp8 quantiser.  Not part of the C ABI.
#ifndef AMULET_EXPERTS_INTERNAL_H
#define AMULET_EXPERTS_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "amulet_internal.h"

namespace amulet {

// types of elements, as in the C ABI (amulet_type_t)
enum { EXPERTS_FP32 = 0, EXPERTS_BF16 = 1, EXPERTS_FP16 = 2, EXPERTS_FP8 = 3,
       EXPERTS_FP8_EXACT = 4 };   // 8-bit operands, their products summed as bf16 ones (experts_mm_fp8_exact.hip)

// A product by groups of rows, checked on the host.  Pitches and strides in elements.
struct ExpertsArgs {
    const void *A, *B;
    void *R;
    const int32_t *offsets;          // G + 1 first rows, or null: one group of all rows
    const int32_t *rows;             // storage row of A (by sums: of A or D) for each row, or null
    const float *scale_a, *scale_b;  // fp8: [k block][row of A]; [block of B's storage rows][block of its columns]
    float *workspace;                // by sums, parts > 1: fp32 sums of tiles
    int64_t lda, ldb, ldr, group_b, group_r, ld_sa, ld_sb, group_sb;
    int M, N, K, G;                  // by sums: M, N are the columns of A's and D's storage
    int a_rows;                      // rows that `rows` may name
    int k_rows;                      // by sums: rows of all groups
    int parts;                       // by sums: ranges of a group's rows, each a workgroup's
    int rows_of_b;                   // by sums: `rows` names D's rows
    int out;                         // type of R
    int part_of, units, gap;         // by rows: EXPERTS_BEFORE or _BEHIND the cut of columns_of_largest(), or all of them (0); what it goes by
};
enum { EXPERTS_BEFORE = 1, EXPERTS_BEHIND = 2 };

// Of `cols` columns of 256 x 256 tiles, `rows` high, those that the 256 x 256 tile takes; 128 x 128 tiles take the others.  All, unless a last
// round of few tiles on `units` compute units would cost more than one round of small tiles for the columns that the full rounds
// leave.  In 256ths of a round: the partly full one takes 0.65 of it, whatever its share (of up to a half; what stands still leaves
// the others more power), the small tiles 0.45, or 0.3 where no unit has two, the second launch `gap`; two rounds of small tiles gain nothing.
// Measured, one launch / two, us: bf16, 4096 x 4608 x 4096 188 / 150 (1.12 rounds), 7000 x 2816 x 2816 over 3 groups 141 / 120 (1.2), 5000 x 4096 x
// 4096 over 4 180 / 166 (1.3), 16384 x 2048 x 4096 over 16 327 / 304 (2.28); with small tiles for more than half a round 6000 x 4096 x 2048 99 / 113 (1.5), after
// short rounds 8192 x 4096 x 1024 over 8 87 / 90 (2.25).  Integers: host and device have to agree.
__host__ __device__ inline int columns_of_largest(int64_t rows, int cols, int units, int gap)
{
    const int64_t tiles = rows * cols, full = tiles / units, rest = tiles - full * units;
    if (full == 0 || rest == 0) return cols;
    const int64_t before = full * units / rows, behind = rows * (cols - before);
    if (before == 0) return cols;
    if (2 * behind > units) return cols;
    const int64_t one = 256 * full + 166, two = 256 * full + (8 * behind <= units ? 77 : 115) + gap;
    return 20 * two < 19 * one ? (int)before : cols;
}

// Of an operand stored across k whose rows of `row` bytes end inside a unit of 16: of its first `whole` stages of bk k, those that may be read by
// whole units.  The last unit of a row reaches past it, into rows that have to be there: of `k`, `pitch` bytes apart, k - whole bk
// lie behind the last one read (rows shorter than a unit may need several).
__host__ __device__ inline int stages_of_whole_units(int whole, int bk, int k, int64_t row, int64_t pitch)
{
    // (one stage fewer is enough: its rows hold more than a unit)
    return whole > 0 && (int64_t)(k - whole * bk) * pitch < 16 - row % 16 ? whole - 1 : whole;
}

// tiles of R by rows (experts_mm_*.hip): rows x columns; _K2: two groups of waves share a tile's k
enum { EXPERTS_256x256 = 0, EXPERTS_128x128 = 1, EXPERTS_64x128 = 2, EXPERTS_64x64 = 3, EXPERTS_64x64_K2 = 4, EXPERTS_16x32 = 5, EXPERTS_TILES = 6 };
constexpr int kExpertsTileRows[EXPERTS_TILES] = {256, 128, 64, 64, 64, 16};
constexpr int kExpertsTileCols[EXPERTS_TILES] = {256, 128, 128, 64, 64, 32};

// `blocks` workgroups of tile shape `tile`; b_across: B's storage has k across its rows (K x N), else N x K
hipError_t launch_experts_rows_bf16(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s);
hipError_t launch_experts_rows_fp16(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s);
hipError_t launch_experts_rows_fp8(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s);
// ... for results of 32 bits; no 256 x 256 tile
hipError_t launch_experts_rows_fp8_exact(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s);
// What a product by rows launches: `blocks` workgroups of `tile` (-1: no launch holds it), and `behind` of EXPERTS_128x128 where those take the last
// columns (a.units and a.gap say which).  first: the largest tile that may be taken.
struct RowsPlan {
    int tile;
    int64_t blocks, behind;
};
RowsPlan rows_plan(int es, bool b_across, ExpertsArgs &a, int64_t M, int64_t N, int64_t G, int first);
// by sums: tile EXPERTS_256x256, EXPERTS_128x128 or EXPERTS_64x64
hipError_t launch_experts_sums(int type, int tile, const ExpertsArgs &a, int64_t blocks, hipStream_t s);
// how its workgroups share the tiles of a group out over the XCDs, and how many there are of them
__host__ __device__ inline bool sums_by_group(int64_t tiles_of_a_group) { return tiles_of_a_group >= 32; }
inline int64_t sums_blocks(int64_t tiles_of_a_group, int64_t pieces)
{
    return 8 * (sums_by_group(tiles_of_a_group) ? (tiles_of_a_group + 7) / 8 * pieces : (tiles_of_a_group * pieces + 7) / 8);
}
// R = the parts' sums, added up in order
hipError_t launch_experts_join(int tile, const ExpertsArgs &a, hipStream_t s);

struct RouteArgs {
    const void *logits; int64_t ldx; int type;
    int T, E, k, norm;
    int32_t *experts, *place, *tokens, *offsets;
    float *weights;
    int32_t *counts;                 // workspace: [block of tokens][expert]
    const float *dweights;           // gradient only
    void *dlogits; int64_t lddx;
};
hipError_t launch_route(const RouteArgs &a, hipStream_t s);
hipError_t launch_route_grad(const RouteArgs &a, hipStream_t s);
// the lanes of a token there: every one has one of the chosen experts; 256 threads to a workgroup
inline int route_grad_lanes(int64_t E, int64_t k) { return k > 16 || E > 256 ? 64 : 16; }
int64_t route_blocks(int64_t T);     // blocks of tokens whose experts are counted apart

struct CombineArgs {
    const void *Y; int64_t ldy;
    const float *weights;            // null: ones
    const int32_t *place;
    void *R; int64_t ldr;            // the sum (gradient: its gradient, read)
    void *dY; int64_t lddy;
    float *dweights;
    int T, k, H, type;
    int64_t rows;                    // of Y
};
hipError_t launch_combine(const CombineArgs &a, hipStream_t s);
hipError_t launch_combine_grad(const CombineArgs &a, hipStream_t s);

struct QuantizeArgs {
    const void *X; int64_t ldx, group_x;
    uint8_t *Q; int64_t ldq, group_q;
    float *scales; int64_t lds, group_s;
    int G, M, K, type;
};
// a scale for each row and 128 columns; for each 128 x 128
hipError_t launch_quantize_rows(const QuantizeArgs &a, hipStream_t s);
hipError_t launch_quantize_blocks(const QuantizeArgs &a, hipStream_t s);

// the calling thread's note of a call (amulet_recent_kernel): what its second launch is, if there is one; and the status of a
// launch's error (amulet_last_launch_error)
void note_kernel(const char *name, int64_t rows, int last_columns = 0, int parts = 1);
int launch_status(hipError_t e);

}  // namespace amulet
#endif
