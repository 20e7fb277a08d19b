// C ABI of a mixture-of-experts layer's operators: argument checks, the choice of tiles, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "amulet.h"
#include "experts_internal.h"

namespace amulet {

static const int64_t kMostRows = 2147483647LL - 65536LL;   // of a dimension, as in the other calls
static const int64_t kMostGroups = 1 << 16;              // (every workgroup looks through the offsets)
static const int64_t kMostBlocks = 0xffffffffLL / 512;     // workgroups of a launch (a grid holds 2^32 - 1 work-items)
static const int64_t kMostBlocks256 = 0xffffffffLL / 256;  // ... of 256 threads

// the longest pitch (bytes) of an operand whose tile's lines, or a stage's k, lie within 32 bits of each other: 256 of them, and a row
static const int64_t kMostPitch = 0xffffffffLL / 256 - 65536;

static bool known16(int type) { return type == AMULET_BF16 || type == AMULET_FP16; }
static bool known(int type) { return type == AMULET_FP32 || known16(type); }

// G matrices of rows x cols, rows ld apart and matrices `group`, that are written: no two share an element.  Either they lie one behind
// the other, or the rows of all of them in turn.
static bool groups_apart(int64_t G, int64_t rows, int64_t cols, int64_t ld, int64_t group)
{
    if (G <= 1) return true;
    return group >= cols && ((group - cols) / ld >= rows - 1 || (ld - cols) / group >= G - 1);
}

// Tiles by rows: the one with the lowest estimate.  A workgroup that has its unit alone takes `stage` us for a stage of its k
// (64 of 16 bits, 128 of 8), of which larger tiles have less per product, and `start` for finding its tile, filling its ring and
// storing; all workgroups together take no more from the L2s than some 64 KB a us and unit, of which smaller tiles
// need more; under both lies what memory takes for the operands, TB/s as a tile's requests draw it (of 16 bits along k,
// across it, of 8 bits).  The numbers were measured, and fitted to 369 sizes (1 ... 32768 rows, widths of 64 to 4096, 1 ... 128 groups, 16
// and 8 bits, both layouts, operands in the caches and out of them): 3 % behind the fastest on average.  us,
// 256 x 256 / 128 x 128 / 64 x 128 / 64 x 64 / 64 x 64 with two k groups / 16 x 32, bf16, B stored N x K: 256 x 4096 x 4096
// 85 / 46 / 28 / 22 / 18 / 38, 64 x 512 x 4096 58 / 42 / 25 / 19 / 14 / 8, 1024 x 4096 x 1024 over 8 groups 26 / 19 / 18 / 19 / 29 / 60, 8192 x 1024 x 1024
// over 8 32 / 26 / 28 / 37 / - / 121, 48 x 2048 x 2048 over 64 (out of memory) 67 / 63 / 59 / 59 / 62 / 51; 4096 x 4096 x 1024 over 4 of 8 bits 30 / 33 / 40 / 46 / 83 / 216.
// It knows nothing of the address of rows and takes 8-bit operands with results of 32 bits, whose stage has four times the instructions, for
// the others of 8 bits: 3001 x 1501 x 1003 over 7 groups, rows at odd addresses, fp16, 14 us where 31 are measured, 1777 x 1368 x 2504 over 5, 8 bits with
// results of 32, 18 where 34 are.
// (Tiles of 16 x 64 and 32 x 64 that were tried gained 0.1 % on average and are not built.)
struct TileCost {
    double stage16, stage8, start;       // us
    double along16, across16, memory8;   // TB/s
    int resident;                        // workgroups that a unit's LDS holds
};
static const TileCost kTileCosts[EXPERTS_TILES] = {
    {1.22, 1.21, 7.9, 4.0, 4.6, 4.0, 1}, {0.67, 0.75, 2.6, 4.5, 5.3, 4.3, 2}, {0.37, 0.86, 2.6, 4.6, 5.1, 4.8, 2},
    {0.30, 0.50, 1.8, 5.1, 4.8, 4.0, 3}, {0.25, 0.39, 3.8, 4.8, 4.7, 3.4, 1}, {0.10, 0.14, 3.7, 5.7, 4.7, 3.5, 2}};
static double tile_us(int tile, int64_t M, int64_t N, int64_t K, int64_t G, int es, bool b_across)
{
    const double units = compute_units(), bm = kExpertsTileRows[tile], bn = kExpertsTileCols[tile];
    const double busy = (double)(G < M ? G : M), per = (double)M / busy;
    // row tiles: a group's last one is half full on average
    const double rows = per <= bm ? busy : G > 1 ? (double)M / bm + 0.5 * busy : (double)((M + (int64_t)bm - 1) / (int64_t)bm);
    const double groups = rows * (double)((N + (int64_t)bn - 1) / (int64_t)bn), stages = (double)((K * es + 127) / 128);
    const TileCost &c = kTileCosts[tile];
    const double round = units * c.resident;
    const double rounds = groups <= round ? 1.0 : groups / round;   // (units take their next tile as they finish)
    const double alone = rounds * (stages * (es == 1 ? c.stage8 : c.stage16) + c.start);
    // (a line of 64 bytes of B across k: two requests for what one brings)
    const double bytes = bm + bn * (b_across && bn * es < 128 ? 2.1 : 1.0);
    const double supply = groups / units * stages * bytes * 0.128 / 64.0;
    const double memory = (busy * (double)N * (double)K + (double)M * (double)K) * es / (1e6 * (es == 1 ? c.memory8 : b_across ? c.across16 : c.along16));
    const double most = alone > supply ? alone : supply;
    return (most > memory ? most : memory) + 0.03 * (alone + supply);
}
// Workgroups that are enough for any offsets: a group's last tile may hold one row only, and the rows outside the groups
// are two regions more.
static int64_t rows_blocks(int tile, int64_t M, int64_t N, int64_t G, bool grouped)
{
    const int64_t bm = kExpertsTileRows[tile], bn = kExpertsTileCols[tile];
    const int64_t regions = !grouped ? 1 : G + 2 < M ? G + 2 : M;
    const int64_t tiles = (M + regions * (bm - 1)) / bm * ((N + bn - 1) / bn);
    return (tiles + 7) / 8 * 8;
}

// The tile with the lowest estimate of those whose workgroups one launch holds; -1: none
static int rows_tile(int64_t M, int64_t N, int64_t K, int64_t G, int es, bool b_across, bool grouped, int first)
{
    int best = -1;
    double least = 0.0;
    for (int tile = EXPERTS_TILES - 1; tile >= first; --tile) {
        if (rows_blocks(tile, M, N, G, grouped) > kMostBlocks) continue;
        const double us = tile_us(tile, M, N, K, G < 1 ? 1 : G, es, b_across);
        if (best < 0 || us < least) { least = us; best = tile; }
    }
    return best;
}

static int check_rows(int es, int64_t M, int64_t N, int64_t K, int64_t G, int trans_b, const void *A, int64_t lda, const int32_t *rows, int64_t a_rows,
                      const void *B, int64_t ldb, int64_t group_b, const int32_t *offsets, bool grouped, const void *R, int64_t ldr)
{
    if (M < 0 || N < 0 || K < 0 || G < 0 || a_rows < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || N > kMostRows || K > kMostRows || a_rows > kMostRows || G > kMostGroups) return AMULET_ERR_RANGE;
    if (M == 0 || N == 0) return 1;   // nothing to write
    if (!R || (grouped && !offsets)) return AMULET_ERR_NULL;
    if (ldr < N) return AMULET_ERR_LD;
    if (K == 0 || G == 0 || (rows && a_rows == 0)) return AMULET_OK;   // zeros: the operands are not read
    if (!A || !B) return AMULET_ERR_NULL;
    if (lda < K || ldb < (trans_b ? K : N) || (G > 1 && group_b < 0)) return AMULET_ERR_LD;
    if (lda > kMostPitch / es || ldb > kMostPitch / es) return AMULET_ERR_RANGE;
    return AMULET_OK;
}

// Workgroups of 128 x 128 tiles for the columns behind the cut of columns_of_largest(), which the kernels make by the rows of tiles that the offsets
// give; 0: one launch for all columns, as the cut is unlikely.  The rows of tiles of random groups lie within some sqrt(G / 3) of what half
// a tile for each group's last makes.
static int64_t cut_blocks(ExpertsArgs &a, int64_t M, int64_t N, int64_t G, bool grouped, int es)
{
    if (G > 128) return 0;   // (last tiles' number too uncertain, and each possible one is looked at)
    const int cols = (int)((N + 255) / 256);
    const double round_us = (double)((a.K * es + 127) / 128) * 1.7 + 8.0;
    a.units = compute_units();
    a.gap = (int)(256.0 * 4.0 / round_us);
    const int64_t least = (M + 255) / 256, regions = G + 2 < M ? G + 2 : M, most = grouped ? (M + regions * 255) / 256 : least;
    const int64_t usual = grouped ? M / 256 + G / 2 : least, spread = grouped ? (int64_t)sqrt((double)G / 3.0) + 1 : 0;
    int64_t blocks = 0;
    int cuts = 0, tried = 0;
    for (int64_t rows = least; rows <= most; ++rows) {
        const int before = columns_of_largest(rows, cols, a.units, a.gap);
        if (rows >= usual - spread && rows <= usual + spread) { ++tried; cuts += before < cols; }
        const int64_t n = 2 * rows * ((N + 127) / 128 - 2 * before);   // (a row of 256 x 256 tiles is at most two of 128 x 128)
        if (before < cols && n > blocks) blocks = n;
    }
    return 2 * cuts > tried ? (blocks + 7) / 8 * 8 : 0;
}

RowsPlan rows_plan(int es, bool b_across, ExpertsArgs &a, int64_t M, int64_t N, int64_t G, int first)
{
    RowsPlan p = {rows_tile(M, N, a.K, G, es, b_across, a.offsets != nullptr, first), 0, 0};
    if (p.tile < 0) return p;
    p.blocks = rows_blocks(p.tile, M, N, G, a.offsets != nullptr);
    p.behind = p.tile == EXPERTS_256x256 ? cut_blocks(a, M, N, G, a.offsets != nullptr, es) : 0;
    return p;
}

static int run_rows(const char *const *names, int type, int trans_b, ExpertsArgs &a, int64_t M, int64_t N, int64_t G, void *stream)
{
    // 8-bit operands whose results keep 32 bits have no 256 x 256 tile, and that tile's offsets of A's rows have 32 bits
    const int es = type == EXPERTS_BF16 || type == EXPERTS_FP16 ? 2 : 1;
    const bool near = (a.rows ? (int64_t)a.a_rows : 256) <= 0xffffffffLL / es / (a.lda > 0 ? a.lda : 1);
    const RowsPlan plan = rows_plan(es, !trans_b, a, M, N, G, type != EXPERTS_FP8_EXACT && near ? EXPERTS_256x256 : EXPERTS_128x128);
    const int tile = plan.tile;
    if (tile < 0) return AMULET_ERR_RANGE;
    const int64_t blocks = plan.blocks, behind = plan.behind;
    note_kernel(names[tile], M, behind ? kExpertsTileCols[EXPERTS_128x128] : 0);
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](int shape, int64_t n) {
        switch (type) {
        case EXPERTS_BF16: return launch_status(launch_experts_rows_bf16(shape, !trans_b, a, n, s));
        case EXPERTS_FP16: return launch_status(launch_experts_rows_fp16(shape, !trans_b, a, n, s));
        case EXPERTS_FP8_EXACT: return launch_status(launch_experts_rows_fp8_exact(shape, !trans_b, a, n, s));
        default: return launch_status(launch_experts_rows_fp8(shape, !trans_b, a, n, s));
        }
    };
    if (behind == 0) return launch(tile, blocks);
    a.part_of = EXPERTS_BEFORE;
    const int rc = launch(tile, blocks);
    if (rc != AMULET_OK) return rc;
    a.part_of = EXPERTS_BEHIND;
    return launch(EXPERTS_128x128, behind);
}

static const char *const kRowsNames[EXPERTS_TILES] = {"grouped_mm_256x256", "grouped_mm_128x128", "grouped_mm_64x128", "grouped_mm_64x64",
                                                      "grouped_mm_64x64_k2", "grouped_mm_16x32"};
static const char *const kFp8Names[EXPERTS_TILES] = {"mm_fp8_256x256", "mm_fp8_128x128", "mm_fp8_64x128", "mm_fp8_64x64",
                                                     "mm_fp8_64x64_k2", "mm_fp8_16x32"};

// The weights' gradients: tiles, and the parts that a group's rows are summed in.  A part is a workgroup of its own that
// writes its fp32 sums to the workspace, which a second kernel adds up: worth it where few outputs have many rows.  The estimate is
// of the same kind as tile_us: a workgroup's stages of 64 rows and its start (stores among it), what the L2s
// supply, what memory takes; fitted to 370 sizes (4 ... 32768 rows, 1 ... 128 groups, up to 64 parts), 2.5 % behind the fastest on
// average.  us, 256 x 256 / 128 x 128 / 64 x 64: 16384 rows over 16 groups of 4096 x 2048 392 / 538 / 765, 24008 over 4 of 384 x 832 in 1 part
// 173 / 124 / 71, in 4 66 / 48 / 50, 18339 over 2 of 2432 x 64 in 8 parts 53 / 39 / 28.
struct SumsPlan {
    int tile, parts;
};
static SumsPlan sums_plan(int64_t rows_r, int64_t cols_r, int64_t G, int64_t M, int out_bytes, size_t bytes)
{
    static const struct { int tile; double stage, start; int resident; } kinds[3] = {{EXPERTS_256x256, 1.2, 7.7, 1}, {EXPERTS_128x128, 0.53, 5.1, 2}, {EXPERTS_64x64, 0.38, 3.7, 3}};
    const double units = compute_units();
    SumsPlan best = {EXPERTS_128x128, 1};
    double least = -1.0;
    for (const auto &k : kinds) {
        const int64_t bm = kExpertsTileRows[k.tile], bn = kExpertsTileCols[k.tile];
        const int64_t of_group = ((rows_r + bm - 1) / bm) * ((cols_r + bn - 1) / bn);
        if (of_group > kMostBlocks / G) continue;   // (no launch holds them, and 64 bits need not)
        const int64_t tiles = of_group * G;
        const int64_t room = (int64_t)(bytes / 4 / (size_t)(bm * bn)) / tiles, most = M / (256 * G) < room ? M / (256 * G) : room;
        for (int64_t parts = 1; parts == 1 || (parts <= most && parts <= 64 && tiles * parts <= 4 * k.resident * (int64_t)units); parts += parts < 8 ? 1 : 4) {
            const double groups = (double)tiles * parts, stages = (double)((M + G * parts * 64 - 1) / (G * parts * 64));
            const double rounds = groups <= units * k.resident ? 1.0 : groups / (units * k.resident);
            const double alone = rounds * (stages * k.stage + k.start);
            const double supply = groups / units * stages * (double)(bm + bn) * 0.128 / 81.0;
            const double memory = ((double)M * (rows_r + cols_r) * 2.0 + (double)G * rows_r * cols_r * out_bytes) / 6.3e6;
            double us = alone > supply ? alone : supply;
            us = (us > memory ? us : memory) + 0.12 * (alone + supply);
            if (parts > 1) us += 2.6 + (double)tiles * bm * bn * 4.0 * parts / 2.8e6;
            if (least < 0 || us < least) { least = us; best = {k.tile, (int)parts}; }
        }
    }
    return best;
}

}  // namespace amulet

using namespace amulet;

extern "C" {

size_t amulet_route_workspace_bytes(int64_t T, int64_t E)
{
    if (T <= 64 || E <= 0 || T > kMostRows || E > 1024) return 0;
    return (size_t)(route_blocks(T) * E * 4);
}

static int check_route(int type, int64_t T, int64_t E, int64_t k, int64_t ldx)
{
    if (!known(type)) return AMULET_ERR_TYPE;
    if (T < 0 || E < 1 || k < 1 || k > E) return AMULET_ERR_DIM;
    if (E > 1024 || k > 64 || T > kMostRows / k) return AMULET_ERR_RANGE;
    if (ldx < E) return AMULET_ERR_LD;
    return AMULET_OK;
}

int amulet_route(int type, int64_t T, int64_t E, int64_t k, const void *logits, int64_t ldx, int norm,
                 int32_t *experts, float *weights, int32_t *place, int32_t *tokens, int32_t *offsets,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_route(type, T, E, k, ldx);
    if (rc != AMULET_OK) return rc;
    if (!offsets || (T > 0 && (!logits || !experts || !weights || !place || !tokens))) return AMULET_ERR_NULL;
    const size_t need = amulet_route_workspace_bytes(T, E);
    if (need > 0 && (!workspace || workspace_bytes < need)) return AMULET_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 3) != 0) return AMULET_ERR_WORKSPACE;
    RouteArgs a = {};
    a.logits = logits; a.ldx = ldx; a.type = type;
    a.T = (int)T; a.E = (int)E; a.k = (int)k; a.norm = norm;
    a.experts = experts; a.weights = weights; a.place = place; a.tokens = tokens; a.offsets = offsets;
    a.counts = (int32_t *)workspace;
    note_kernel("route", T);
    return launch_status(launch_route(a, (hipStream_t)stream));
}

int amulet_route_grad(int type, int64_t T, int64_t E, int64_t k, const void *logits, int64_t ldx, int norm,
                      const int32_t *experts, const float *weights, const float *dweights,
                      void *dlogits, int64_t lddx, void *stream)
{
    const int rc = check_route(type, T, E, k, norm ? E : ldx);
    if (rc != AMULET_OK) return rc;
    if (T == 0) return AMULET_OK;
    if ((T - 1) / (route_grad_lanes(E, k) == 16 ? 16 : 4) >= kMostBlocks256) return AMULET_ERR_RANGE;
    if ((!norm && !logits) || !experts || !weights || !dweights || !dlogits) return AMULET_ERR_NULL;
    if (lddx < E) return AMULET_ERR_LD;
    RouteArgs a = {};
    a.logits = logits; a.ldx = ldx; a.type = type;
    a.T = (int)T; a.E = (int)E; a.k = (int)k; a.norm = norm;
    a.experts = (int32_t *)experts; a.weights = (float *)weights; a.dweights = dweights;
    a.dlogits = dlogits; a.lddx = lddx;
    note_kernel("route_grad", T);
    return launch_status(launch_route_grad(a, (hipStream_t)stream));
}

static int check_combine(int type, int64_t T, int64_t k, int64_t H, int64_t rows, bool grad)
{
    if (!known(type)) return AMULET_ERR_TYPE;
    if (T < 0 || k < 0 || H < 0 || rows < 0) return AMULET_ERR_DIM;
    if (H > kMostRows || rows > kMostRows || k > kMostRows || T > kMostRows / (k > 0 ? k : 1)) return AMULET_ERR_RANGE;
    if (T == 0 || H == 0) return 1;
    // (four waves to a workgroup: each has 16 bytes to a lane of a token's columns, backward a pair)
    const int64_t columns = type == AMULET_FP32 ? 256 : 512, waves = T * (grad ? k : (H + columns - 1) / columns);
    return (waves + 3) / 4 > kMostBlocks256 ? AMULET_ERR_RANGE : AMULET_OK;
}

int amulet_combine(int type, int64_t T, int64_t k, int64_t H, int64_t rows, const void *Y, int64_t ldy,
                   const float *weights, const int32_t *place, void *R, int64_t ldr, void *stream)
{
    const int rc = check_combine(type, T, k, H, rows, false);
    if (rc != AMULET_OK) return rc > 0 ? AMULET_OK : rc;
    if (!R || (k > 0 && !place) || (k > 0 && rows > 0 && !Y)) return AMULET_ERR_NULL;
    if (ldr < H || (k > 0 && rows > 0 && ldy < H)) return AMULET_ERR_LD;
    CombineArgs a = {};
    a.Y = Y; a.ldy = ldy; a.weights = weights; a.place = place; a.R = R; a.ldr = ldr;
    a.T = (int)T; a.k = (int)k; a.H = (int)H; a.type = type; a.rows = rows;
    note_kernel("combine", T);
    return launch_status(launch_combine(a, (hipStream_t)stream));
}

int amulet_combine_grad(int type, int64_t T, int64_t k, int64_t H, int64_t rows, const void *Y, int64_t ldy,
                        const float *weights, const int32_t *place, const void *dR, int64_t lddr,
                        void *dY, int64_t lddy, float *dweights, void *stream)
{
    const int rc = check_combine(type, T, k, H > 0 ? H : 1, rows, true);
    if (rc != AMULET_OK) return rc > 0 ? AMULET_OK : rc;
    if (H < 0) return AMULET_ERR_DIM;
    if (k == 0) return AMULET_OK;
    if (!place || (H > 0 && (!dR || (rows > 0 && (!dY || (dweights && !Y)))))) return AMULET_ERR_NULL;
    if (lddr < H || (rows > 0 && (lddy < H || (dweights && ldy < H)))) return AMULET_ERR_LD;
    CombineArgs a = {};
    a.Y = Y; a.ldy = ldy; a.weights = weights; a.place = place; a.R = (void *)dR; a.ldr = lddr;
    a.dY = dY; a.lddy = lddy; a.dweights = dweights;
    a.T = (int)T; a.k = (int)k; a.H = (int)H; a.type = type; a.rows = rows;
    note_kernel("combine_grad", T);
    return launch_status(launch_combine_grad(a, (hipStream_t)stream));
}

int amulet_grouped_mm(int type, int out_type, int trans_b, int64_t M, int64_t N, int64_t K, int64_t G,
                      const void *A, int64_t lda, const int32_t *rows, int64_t a_rows,
                      const void *B, int64_t ldb, int64_t group_b, const int32_t *offsets,
                      void *R, int64_t ldr, void *stream)
{
    if (!known16(type) || (out_type != AMULET_FP32 && out_type != type)) return AMULET_ERR_TYPE;
    const int rc = check_rows(2, M, N, K, G, trans_b, A, lda, rows, a_rows, B, ldb, group_b, offsets, true, R, ldr);
    if (rc != AMULET_OK) return rc > 0 ? AMULET_OK : rc;
    ExpertsArgs a = {};
    a.A = A; a.B = B; a.R = R; a.offsets = offsets; a.rows = rows;
    a.lda = lda; a.ldb = ldb; a.ldr = ldr; a.group_b = group_b;
    a.M = (int)M; a.N = (int)N; a.K = G == 0 || (rows && a_rows == 0) ? 0 : (int)K; a.G = (int)G; a.a_rows = (int)a_rows;
    a.out = out_type;
    return run_rows(kRowsNames, type, trans_b, a, M, N, G, stream);
}

size_t amulet_grouped_mm_wgrad_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t G)
{
    if (M <= 0 || N <= 0 || K <= 0 || G <= 0 || M > kMostRows || N > kMostRows || K > kMostRows || G > kMostGroups) return 0;
    size_t most = 0;
    for (int out_bytes = 2; out_bytes <= 4; out_bytes += 2) {   // (R's type is not known here)
        const SumsPlan plan = sums_plan(K, N, G, M, out_bytes, ~(size_t)0 >> 1);
        const int64_t bm = kExpertsTileRows[plan.tile], bn = kExpertsTileCols[plan.tile];
        const size_t bytes = plan.parts < 2 ? 0 : (size_t)(((K + bm - 1) / bm) * ((N + bn - 1) / bn) * G * plan.parts * bm * bn * 4);
        if (bytes > most) most = bytes;
    }
    return most;
}

int amulet_grouped_mm_wgrad(int type, int out_type, int trans_r, int64_t M, int64_t N, int64_t K, int64_t G,
                            const void *A, int64_t lda, const int32_t *rows, int64_t a_rows,
                            const void *D, int64_t ldd, const int32_t *offsets,
                            void *R, int64_t ldr, int64_t group_r,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    if (!known16(type) || (out_type != AMULET_FP32 && out_type != type)) return AMULET_ERR_TYPE;
    if (M < 0 || N < 0 || K < 0 || G < 0 || a_rows < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || N > kMostRows || K > kMostRows || a_rows > kMostRows || G > kMostGroups) return AMULET_ERR_RANGE;
    if (G == 0 || N == 0 || K == 0) return AMULET_OK;
    if (!R || !offsets) return AMULET_ERR_NULL;
    if (ldr < (trans_r ? K : N) || !groups_apart(G, trans_r ? N : K, trans_r ? K : N, ldr, group_r)) return AMULET_ERR_LD;
    const bool some = M > 0 && !(rows && a_rows == 0);   // else: zeros, and the operands are not read
    if (some && (!A || !D)) return AMULET_ERR_NULL;
    if (some && (lda < K || ldd < N)) return AMULET_ERR_LD;
    if (some && (lda > kMostPitch / 2 || ldd > kMostPitch / 2)) return AMULET_ERR_RANGE;
    ExpertsArgs a = {};
    a.R = R; a.offsets = offsets; a.rows = rows; a.ldr = ldr; a.group_r = group_r;
    a.G = (int)G; a.a_rows = (int)a_rows; a.k_rows = some ? (int)M : 0; a.out = out_type;
    // lines of the first operand are R's rows
    if (trans_r) { a.A = D; a.lda = ldd; a.B = A; a.ldb = lda; a.M = (int)N; a.N = (int)K; a.rows_of_b = 1; }
    else { a.A = A; a.lda = lda; a.B = D; a.ldb = ldd; a.M = (int)K; a.N = (int)N; }
    if (((uintptr_t)workspace & 15) != 0) return AMULET_ERR_WORKSPACE;
    a.workspace = (float *)workspace;
    const SumsPlan plan = sums_plan(a.M, a.N, G, M, out_type == AMULET_FP32 ? 4 : 2, workspace ? workspace_bytes : 0);
    const int tile = plan.tile;
    a.parts = plan.parts;
    const int64_t bm = kExpertsTileRows[tile], bn = kExpertsTileCols[tile];
    const int64_t of_group = ((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn);
    if (of_group > kMostBlocks / G) return AMULET_ERR_RANGE;
    const int64_t tiles = of_group * G;
    // (with several parts, which are not for many tiles, the second launch has a workgroup to 1024 outputs)
    if (sums_blocks(of_group, G * a.parts) > kMostBlocks || (a.parts > 1 && tiles * (bm * bn / 1024) > kMostBlocks)) return AMULET_ERR_RANGE;
    note_kernel(tile == EXPERTS_256x256 ? "grouped_mm_wgrad_256x256" : tile == EXPERTS_128x128 ? "grouped_mm_wgrad_128x128" : "grouped_mm_wgrad_64x64", M, 0, a.parts);
    hipStream_t s = (hipStream_t)stream;
    const int rc = launch_status(launch_experts_sums(type, tile, a, sums_blocks(of_group, G * a.parts), s));
    if (rc != AMULET_OK || a.parts == 1) return rc;
    return launch_status(launch_experts_join(tile, a, s));
}

int amulet_quantize_fp8(int type, int64_t M, int64_t K, const void *X, int64_t ldx,
                        void *Q, int64_t ldq, float *scales, int64_t lds, void *stream)
{
    if (!known(type)) return AMULET_ERR_TYPE;
    if (M < 0 || K < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || K > kMostRows || (M + 15) / 16 * ((K + 511) / 512) > kMostBlocks256) return AMULET_ERR_RANGE;
    if (M == 0 || K == 0) return AMULET_OK;
    if (!X || !Q || !scales) return AMULET_ERR_NULL;
    if (ldx < K || ldq < K || lds < M) return AMULET_ERR_LD;
    QuantizeArgs a = {};
    a.X = X; a.ldx = ldx; a.Q = (uint8_t *)Q; a.ldq = ldq; a.scales = scales; a.lds = lds;
    a.G = 1; a.M = (int)M; a.K = (int)K; a.type = type;
    note_kernel("quantize_fp8", M);
    return launch_status(launch_quantize_rows(a, (hipStream_t)stream));
}

int amulet_quantize_fp8_blocks(int type, int64_t G, int64_t M, int64_t K, const void *X, int64_t ldx, int64_t group_x,
                               void *Q, int64_t ldq, int64_t group_q, float *scales, int64_t lds, int64_t group_s,
                               void *stream)
{
    if (!known(type)) return AMULET_ERR_TYPE;
    if (G < 0 || M < 0 || K < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || K > kMostRows || G > kMostGroups) return AMULET_ERR_RANGE;
    if (G == 0 || M == 0 || K == 0) return AMULET_OK;
    const int64_t MB = (M + 127) / 128, KB = (K + 127) / 128;
    if (MB * KB > kMostBlocks / G) return AMULET_ERR_RANGE;
    if (!X || !Q || !scales) return AMULET_ERR_NULL;
    if (ldx < K || ldq < K || lds < KB || (G > 1 && group_x < 0)) return AMULET_ERR_LD;
    if (!groups_apart(G, M, K, ldq, group_q) || !groups_apart(G, MB, KB, lds, group_s)) return AMULET_ERR_LD;
    QuantizeArgs a = {};
    a.X = X; a.ldx = ldx; a.group_x = group_x; a.Q = (uint8_t *)Q; a.ldq = ldq; a.group_q = group_q;
    a.scales = scales; a.lds = lds; a.group_s = group_s;
    a.G = (int)G; a.M = (int)M; a.K = (int)K; a.type = type;
    note_kernel("quantize_fp8_blocks", G * M);
    return launch_status(launch_quantize_blocks(a, (hipStream_t)stream));
}

static int run_fp8(int out_type, int trans_b, int64_t M, int64_t N, int64_t K, int64_t G,
                   const void *A, int64_t lda, const float *scales_a, int64_t lds_a, const int32_t *rows, int64_t a_rows,
                   const void *B, int64_t ldb, int64_t group_b, const float *scales_b, int64_t lds_b, int64_t group_sb,
                   const int32_t *offsets, bool grouped, void *R, int64_t ldr, void *stream)
{
    if (!known(out_type)) return AMULET_ERR_TYPE;
    const int rc = check_rows(1, M, N, K, G, trans_b, A, lda, rows, a_rows, B, ldb, group_b, offsets, grouped, R, ldr);
    if (rc != AMULET_OK) return rc > 0 ? AMULET_OK : rc;
    const bool some = K > 0 && G > 0 && !(rows && a_rows == 0);
    if (some && (rows ? a_rows : M) > (1 << 30)) return AMULET_ERR_RANGE;   // (32-bit byte offsets of a block's scales)
    if (some && (!scales_a || !scales_b)) return AMULET_ERR_NULL;
    if (some && (lds_a < (rows ? a_rows : M) || lds_b < ((trans_b ? K : N) + 127) / 128 || (G > 1 && group_sb < 0))) return AMULET_ERR_LD;
    ExpertsArgs a = {};
    a.A = A; a.B = B; a.R = R; a.offsets = offsets; a.rows = rows; a.scale_a = scales_a; a.scale_b = scales_b;
    a.lda = lda; a.ldb = ldb; a.ldr = ldr; a.group_b = group_b; a.ld_sa = lds_a; a.ld_sb = lds_b; a.group_sb = group_sb;
    a.M = (int)M; a.N = (int)N; a.K = some ? (int)K : 0; a.G = (int)G; a.a_rows = (int)a_rows;
    a.out = out_type;
    return run_rows(kFp8Names, out_type == AMULET_FP32 ? EXPERTS_FP8_EXACT : EXPERTS_FP8, trans_b, a, M, N, G, stream);
}

int amulet_grouped_mm_fp8(int out_type, int trans_b, int64_t M, int64_t N, int64_t K, int64_t G,
                          const void *A, int64_t lda, const float *scales_a, int64_t lds_a, const int32_t *rows, int64_t a_rows,
                          const void *B, int64_t ldb, int64_t group_b, const float *scales_b, int64_t lds_b, int64_t group_sb,
                          const int32_t *offsets, void *R, int64_t ldr, void *stream)
{
    return run_fp8(out_type, trans_b, M, N, K, G, A, lda, scales_a, lds_a, rows, a_rows, B, ldb, group_b, scales_b, lds_b, group_sb, offsets, true, R, ldr, stream);
}

int amulet_mm_fp8(int out_type, int trans_b, int64_t M, int64_t N, int64_t K,
                  const void *A, int64_t lda, const float *scales_a, int64_t lds_a,
                  const void *B, int64_t ldb, const float *scales_b, int64_t lds_b,
                  void *R, int64_t ldr, void *stream)
{
    return run_fp8(out_type, trans_b, M, N, K, 1, A, lda, scales_a, lds_a, nullptr, 0, B, ldb, 0, scales_b, lds_b, 0, nullptr, false, R, ldr, stream);
}

}  // extern "C"
