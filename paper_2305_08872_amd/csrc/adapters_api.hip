// C ABI of the low-rank adapters and of the gradients' norm: argument checks, choices, launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "adapters_internal.h"
#include "amulet.h"

namespace amulet {

static const int64_t kMostRows = 2147483647LL - 65536LL;   // of a dimension, as in the other calls
static const int64_t kMostGroups = 1 << 16;                // adapters, and segments
static const int64_t kMostRank = 1 << 16;
static const int64_t kMostBlocks256 = 0xffffffffLL / 256;  // workgroups of a launch (a grid holds 2^32 - 1 work-items) of 256 threads
static const int64_t kMostPitch = 0xffffffffLL / 256 - 65536;   // bytes, of the shared product's operands (as in the products by groups)

static bool known16(int type) { return type == AMULET_BF16 || type == AMULET_FP16; }

static const char *const kUpNames[ADAPTERS_16x16 + 1] = {"adapters_256x256", "adapters_128x128", "adapters_64x128", "adapters_64x64", "adapters_64x64_k2", "adapters_16x32",
                                                         "adapters_16x16"};

// G matrices of rows x cols that are written: no two share an element, one behind the other or their rows in turn
static bool matrices_apart(int64_t G, int64_t rows, int64_t cols, int64_t ld, int64_t group)
{
    if (G <= 1) return true;
    return group >= cols && ((group - cols) / ld >= rows - 1 || (ld - cols) / group >= G - 1);
}

// How the gradients' sums are shared out.  Columns to a workgroup: 128, or 64 (half of a row's bytes in a request) where those would not
// give every compute unit one.  Rows: an adapter's, or pieces of it, two workgroups of four waves to a compute unit, that the workspace has
// room for, of 512 rows at least (fewer are not worth the second launch, 4 us).  us, whole / pieces of 512 / 1024 / 2048 rows, out of the caches
// (rank 16, here and below: T in two pieces, 1 us less than three):
// 16384 x 4096 by rank 16, 4 adapters of equal rows 42 / 37 / 34 / 33, one of them with half of the rows 73 / 39 / 41 / 40; 4096 x 4096 by rank 64,
// 8 adapters, results of 32 bits 20 / 24 / 24 / 24 and 45 / 31 / 29 / 43.
struct OuterPlan {
    int columns, quota;
    int64_t pieces;
};
static OuterPlan outer_plan(int64_t M, int64_t N, int64_t r, int64_t G, size_t bytes)
{
    const int64_t units = compute_units(), ranks = r <= 16 ? 1 : (r + 31) / 32, wide = (N + 127) / 128 * ranks;
    OuterPlan p = {wide * G >= units || M >= 512 * 2 * G ? 128 : 64, 0, G};
    const int64_t blocks = (N + p.columns - 1) / p.columns * ranks;
    // Pieces: as many as two workgroups to a compute unit make, or twice that, of which each adapter may leave one that is not full; with as many
    // adapters, no more than keep one that has most rows from being the last.  us, of 16384 rows, 4096 columns, 4 adapters: rank 16, quota 512 / 1024 /
    // 1366 42 / 39 / 36, rank 64 80 / 72 / 66.
    const int64_t fill = 2 * units / blocks, least = 512;
    const int64_t full = G >= fill ? fill : (3 * G <= fill ? fill : 2 * fill) - G;
    int64_t quota = full > 0 ? (M + full - 1) / full : M;
    if (quota < least) quota = least;
    if (quota <= 0 || G > kOuterAdapters || M < 2 * quota) return p;
    const int64_t pieces = M / quota + G;
    if ((size_t)pieces > bytes / 4 / (size_t)(N * r)) return p;
    p.quota = (int)quota;
    p.pieces = pieces;
    return p;
}

static int check_tensors(int64_t n, const int32_t *types, const int64_t *counts, const void *const *in, void *const *out)
{
    if (n < 0) return AMULET_ERR_DIM;
    if (n > kMostRows) return AMULET_ERR_RANGE;
    if (n > 0 && (!types || !counts || !in)) return AMULET_ERR_NULL;
    for (int64_t i = 0; i < n; ++i) {
        if (types[i] != AMULET_FP32 && !known16(types[i])) return AMULET_ERR_TYPE;
        if (counts[i] < 0) return AMULET_ERR_DIM;
        if (counts[i] >= (int64_t)1 << 40) return AMULET_ERR_RANGE;
        if (counts[i] > 0 && (!in[i] || (out && !out[i]))) return AMULET_ERR_NULL;
        if (((uint64_t)in[i] | (out ? (uint64_t)out[i] : 0)) >> 48) return AMULET_ERR_RANGE;   // (no address that a GPU has)
    }
    return AMULET_OK;
}

// The next tensors that a launch holds, from *at on (empty ones are passed over); back: from *at down, to below 0
static NormTensors next_tensors(int64_t n, const int32_t *types, const int64_t *counts, const void *const *in, void *const *out, int64_t *at, bool back)
{
    NormTensors t;
    t.n = 0;
    // Chunks: small ones where they are few (a workgroup each), larger ones where a workgroup has several (which it finds one after the other)
    int64_t all = 0, chunks = 0;
    for (int64_t i = *at, some = 0; i >= 0 && i < n && some < NORM_TENSORS; i += back ? -1 : 1) { all += counts[i]; some += counts[i] > 0; }
    t.chunk = kNormChunk;
    while (t.chunk < 8 * kNormChunk && all / t.chunk > 4 * NORM_BLOCKS) t.chunk *= 2;
    for (; *at >= 0 && *at < n && t.n < NORM_TENSORS; *at += back ? -1 : 1) {
        const int64_t i = *at;
        if (counts[i] == 0) continue;
        const int64_t more = (counts[i] + t.chunk - 1) / t.chunk;
        if (t.n > 0 && chunks + more > 0x7fffffffLL) break;
        const uint64_t from = (uint64_t)in[i], to = out ? (uint64_t)out[i] : from;
        t.in[t.n] = (uint32_t)from;
        t.in_upper[t.n] = (uint16_t)(from >> 32);
        t.out[t.n] = (uint32_t)to;
        t.out_upper[t.n] = (uint16_t)(to >> 32);
        t.count[t.n] = (uint32_t)counts[i];
        t.more[t.n] = (uint16_t)((counts[i] >> 32) | types[i] << 8);
        t.first[t.n] = (uint32_t)chunks;
        chunks += more;
        ++t.n;
    }
    t.chunks = (uint32_t)chunks;
    return t;
}
// A workgroup to a chunk, or as many as the chip holds at a time (four to a compute unit), each with every so many chunks: 2048 would be a round and a half,
// 2^28 bf16 values 141 us in place of 119.
static int norm_blocks(const NormTensors &t) { return t.chunks <= NORM_BLOCKS ? (int)t.chunks : NORM_BLOCKS / 2; }

// The launches of the sums; how many sums they leave, or a negative status
static int64_t run_sums(int64_t n, const int32_t *types, const int64_t *counts, const void *const *in, double *sums, hipStream_t s)
{
    int64_t made = 0;
    for (int64_t at = 0; at < n;) {
        const NormTensors t = next_tensors(n, types, counts, in, nullptr, &at, false);
        if (t.n == 0) break;
        const int blocks = norm_blocks(t), rc = launch_status(launch_norm_sums(t, sums + made, blocks, s));
        if (rc != AMULET_OK) return rc;
        made += blocks;
    }
    return made;
}
static int run_clip(int64_t n, const int32_t *types, const int64_t *counts, const void *const *in, void *const *out, NormArgs a, hipStream_t s)
{
    // (from the last tensor on: it is the one that the caches hold)
    bool first = true;
    for (int64_t at = n - 1; at >= 0 || first;) {
        const NormTensors t = next_tensors(n, types, counts, in, out, &at, true);
        if (t.n == 0 && !(first && !a.given)) break;
        const int rc = launch_status(launch_norm_clip(t, a, t.n ? norm_blocks(t) : 1, s));
        if (rc != AMULET_OK) return rc;
        a.given = 1;   // (the first launch has written it)
        first = false;
    }
    return AMULET_OK;
}

}  // namespace amulet

using namespace amulet;

extern "C" {

int amulet_adapters_mm(int type, int out_type, int trans_w, int trans_a, int trans_b, int64_t M, int64_t N, int64_t K, int64_t r, int64_t S, int64_t G,
                       const void *X, int64_t ldx, const void *W, int64_t ldw,
                       const void *A, int64_t lda, int64_t group_a, const void *B, int64_t ldb, int64_t group_b,
                       const int32_t *offsets, const int32_t *adapters, const float *scales,
                       float *T, int64_t ldt, void *R, int64_t ldr, void *stream)
{
    if (!known16(type) || (out_type != AMULET_FP32 && out_type != type)) return AMULET_ERR_TYPE;
    if (M < 0 || N < 0 || K < 0 || r < 0 || S < 0 || G < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || N > kMostRows || K > kMostRows || r > kMostRank || S > kMostGroups || G > kMostGroups) return AMULET_ERR_RANGE;
    if (!adapters && S != G && S > 0) return AMULET_ERR_DIM;
    if (M == 0 || (N == 0 && r == 0)) return AMULET_OK;   // nothing to write
    if ((N > 0 && !R) || (r > 0 && !T)) return AMULET_ERR_NULL;
    if (ldr < N || ldt < r) return AMULET_ERR_LD;
    const bool some = r > 0 && S > 0 && G > 0;            // else: T is zeros, and the adapters' matrices are not read
    if (some && (!offsets || (K > 0 && !A) || (N > 0 && !B))) return AMULET_ERR_NULL;
    if (K > 0 && ((W && N > 0) || some)) {
        if (!X) return AMULET_ERR_NULL;
        if (ldx < K) return AMULET_ERR_LD;
        if (ldx > kMostPitch / 2) return AMULET_ERR_RANGE;
    }
    if (W && K > 0 && N > 0) {
        if (ldw < (trans_w ? K : N)) return AMULET_ERR_LD;
        if (ldw > kMostPitch / 2) return AMULET_ERR_RANGE;
    }
    if (some && K > 0 && (lda < (trans_a ? K : r) || (G > 1 && group_a < 0))) return AMULET_ERR_LD;
    if (some && K > 0 && lda > kMostPitch / 2) return AMULET_ERR_RANGE;
    if (some && N > 0 && (ldb < (trans_b ? r : N) || (G > 1 && group_b < 0))) return AMULET_ERR_LD;
    if (some && N > 0 && ldb > kMostPitch / 2) return AMULET_ERR_RANGE;

    Segments rows = {};
    rows.offsets = offsets; rows.adapters = adapters;
    rows.S = some ? (int)S : 0; rows.G = some ? (int)G : 0; rows.M = (int)M;
    // Segments of a few rows: row by row, which the larger tiles have no room for.  us without the first product, row by row / through LDS, 1, 2, 4 and 8 rows to a
    // segment: 1337 x 3033 x 2319 rank 32 76 / 132, 74 / 89, 73 / 72 and 72 / 59, rank 8 75 / 84, 73 / 64, 71 / 56 and 71 / 51; B across, rank 32, 94 / 173, 92 / 110,
    // 92 / 84 and 92 / 66 (LDS at 1 and 2 rows: T in two pieces, less than three take).  Segments shorter than a block of rows: no more than 64 of those to a tile (4 rows to a
    // segment, B across, 84; 128 rows to a tile, two pieces, 130).
    bool many = some && M < 4 * S;
    const bool brief = some && M < 16 * S;
    UpArgs u = {};
    RowsPlan plan = {};
    if (N > 0) {
        u.mm.A = X; u.mm.lda = ldx; u.mm.B = W; u.mm.ldb = ldw; u.mm.R = R; u.mm.ldr = ldr;
        u.mm.M = (int)M; u.mm.N = (int)N; u.mm.K = W ? (int)K : 0; u.mm.G = 1; u.mm.out = out_type;
        u.rows = rows; u.T = T; u.ldt = ldt; u.B = B; u.ldb = ldb; u.group_b = group_b; u.r = (int)r; u.across = !trans_b;
        plan = rows_plan(2, !trans_w, u.mm, M, N, 1, many ? EXPERTS_64x64 : brief ? EXPERTS_64x128 : EXPERTS_256x256);
        if (plan.tile < 0 && brief) { many = false; plan = rows_plan(2, !trans_w, u.mm, M, N, 1, EXPERTS_256x256); }
        if (plan.tile < 0) return AMULET_ERR_RANGE;
        // Longer segments, and B across, in odd ranks or read more than twice: rather the tile without k groups, through LDS.  (208 x 4096 x 4096, 64 rows to a
        // segment, B across, rank 8 / 32 / 64 24 / 26 / 29 us, row by row 28 / 29 / 38; 8 rows to a segment, row by row, 26 / 27 / 36, through LDS 25 / 32 / 42.)
        if (some && M >= 12 * S && plan.tile == EXPERTS_64x64_K2 && (!trans_b || r % 8 != 0 || r > 64)) plan.tile = EXPERTS_64x64;   // (of as many workgroups)
        // (row by row two columns of B across are read at a time)
        if (some && N < 2 && !trans_b) {
            many = false;
            plan = {EXPERTS_64x64, ((M + 63) / 64 + 7) / 8 * 8, 0};
            if (plan.blocks > kMostBlocks256) return AMULET_ERR_RANGE;
        }
        // One row of tiles that would leave compute units without one: narrower tiles, whose eight k groups have more of W on its way
        if (plan.tile == EXPERTS_16x32 && M <= 16 && (N + 31) / 32 < compute_units()) plan = {ADAPTERS_16x16, (N + 15) / 16 + 7 & ~(int64_t)7, 0};
    }
    hipStream_t s = (hipStream_t)stream;
    if (r > 0) {
        DownArgs d = {};
        d.rows = rows; d.X = X; d.A = A; d.scales = scales; d.T = T;
        d.ldx = ldx; d.lda = lda; d.group_a = group_a; d.ldt = ldt; d.K = (int)K; d.r = (int)r; d.across = !trans_a;
        if (N == 0) note_kernel("adapters_down", M);
        const hipError_t e = launch_adapters_down(type, d, s);
        if (e == hipErrorInvalidConfiguration) return AMULET_ERR_RANGE;
        const int rc = launch_status(e);
        if (rc != AMULET_OK) return rc;
    }
    if (N == 0) return AMULET_OK;
    note_kernel(kUpNames[plan.tile], M, plan.behind ? kExpertsTileCols[EXPERTS_128x128] : 0);
    auto launch = [&](int tile, int64_t blocks) {
        return launch_status(type == AMULET_BF16 ? launch_adapters_up_bf16(tile, !trans_w, many, u, blocks, s) : launch_adapters_up_fp16(tile, !trans_w, many, u, blocks, s));
    };
    if (plan.behind == 0) return launch(plan.tile, plan.blocks);
    u.mm.part_of = EXPERTS_BEFORE;
    const int rc = launch(plan.tile, plan.blocks);
    if (rc != AMULET_OK) return rc;
    u.mm.part_of = EXPERTS_BEHIND;
    return launch(EXPERTS_128x128, plan.behind);
}

size_t amulet_adapters_wgrad_workspace_bytes(int64_t M, int64_t N, int64_t r, int64_t G)
{
    if (M <= 0 || N <= 0 || r <= 0 || G <= 0 || M > kMostRows || N > kMostRows || r > kMostRank || G > kMostGroups) return 0;
    const OuterPlan p = outer_plan(M, N, r, G, ~(size_t)0 >> 1);
    return p.quota == 0 ? 0 : (size_t)p.pieces * (size_t)N * (size_t)r * 4;
}

int amulet_adapters_wgrad(int type, int out_type, int trans_r, int64_t M, int64_t N, int64_t r, int64_t S, int64_t G,
                          const void *X, int64_t ldx, const float *T, int64_t ldt,
                          const int32_t *offsets, const int32_t *adapters, void *R, int64_t ldr, int64_t group_r,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    if (!known16(type) || (out_type != AMULET_FP32 && out_type != type)) return AMULET_ERR_TYPE;
    if (M < 0 || N < 0 || r < 0 || S < 0 || G < 0) return AMULET_ERR_DIM;
    if (M > kMostRows || N > kMostRows || r > kMostRank || S > kMostGroups || G > kMostGroups) return AMULET_ERR_RANGE;
    if (!adapters && S != G && S > 0) return AMULET_ERR_DIM;
    if (G == 0 || N == 0 || r == 0) return AMULET_OK;
    if (!R || (S > 0 && M > 0 && (!offsets || !X || !T))) return AMULET_ERR_NULL;
    if (ldr < (trans_r ? N : r) || !matrices_apart(G, trans_r ? r : N, trans_r ? N : r, ldr, group_r)) return AMULET_ERR_LD;
    if (S > 0 && M > 0 && (ldx < N || ldt < r)) return AMULET_ERR_LD;
    if (S > 0 && M > 0 && (ldx > kMostPitch / 2 || ldt > kMostPitch / 4)) return AMULET_ERR_RANGE;
    if (((uintptr_t)workspace & 15) != 0) return AMULET_ERR_WORKSPACE;
    OuterArgs a = {};
    a.rows.offsets = offsets; a.rows.adapters = adapters;
    a.rows.S = M > 0 ? (int)S : 0; a.rows.G = (int)G; a.rows.M = (int)M;
    a.X = X; a.ldx = ldx; a.T = T; a.ldt = ldt; a.R = R; a.ldr = ldr; a.group_r = group_r; a.workspace = (float *)workspace;
    a.N = (int)N; a.r = (int)r; a.out = out_type; a.trans_r = trans_r != 0;
    if ((N + 63) / 64 > (kMostBlocks256 / ((r + 15) / 16) - 8) / (G + M / 512) || G * (trans_r ? r * ((N + 3) / 4) : N * ((r + 3) / 4)) > kMostBlocks256 * 256)
        return AMULET_ERR_RANGE;
    const OuterPlan p = outer_plan(M, N, r, G, workspace ? workspace_bytes : 0);
    a.columns = p.columns;
    a.quota = p.quota;
    a.pieces = (int)p.pieces;
    note_kernel("adapters_wgrad", M, 0, p.quota > 0 ? 2 : 1);
    hipStream_t s = (hipStream_t)stream;
    const int rc = launch_status(launch_adapters_outer(type, a, s));
    if (rc != AMULET_OK || p.quota == 0) return rc;
    return launch_status(launch_adapters_join(a, s));
}

size_t amulet_grad_norm_workspace_bytes(int64_t n)
{
    if (n <= 0 || n > kMostRows) return 0;
    return (size_t)((n + NORM_TENSORS - 1) / NORM_TENSORS) * NORM_BLOCKS * 8;
}

// (what the sums of n tensors need of it)
static int check_workspace(int64_t n, const void *workspace, size_t bytes)
{
    return n > 0 && (!workspace || ((uintptr_t)workspace & 7) != 0 || bytes < amulet_grad_norm_workspace_bytes(n)) ? AMULET_ERR_WORKSPACE : AMULET_OK;
}

int amulet_grad_norm(int64_t n, const int32_t *types, const int64_t *counts, const void *const *grads, float *norm,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_tensors(n, types, counts, grads, nullptr);
    if (rc != AMULET_OK) return rc;
    if (!norm) return AMULET_ERR_NULL;
    rc = check_workspace(n, workspace, workspace_bytes);
    if (rc != AMULET_OK) return rc;
    note_kernel("grad_norm", n);
    hipStream_t s = (hipStream_t)stream;
    const int64_t made = run_sums(n, types, counts, grads, (double *)workspace, s);
    if (made < 0) return (int)made;
    NormArgs a = {(double *)workspace, (int)made, norm, 0.0f, 0};
    return launch_status(launch_norm_join(a, s));
}

int amulet_grad_clip(int64_t n, const int32_t *types, const int64_t *counts, const void *const *grads, void *const *outs, float max_norm,
                     const float *norm, void *stream)
{
    const int rc = check_tensors(n, types, counts, grads, outs);
    if (rc != AMULET_OK) return rc;
    if (!(max_norm >= 0.0f)) return AMULET_ERR_RANGE;
    if (n == 0) return AMULET_OK;
    if (!norm) return AMULET_ERR_NULL;
    note_kernel("grad_clip", n);
    const NormArgs a = {nullptr, 0, (float *)norm, max_norm, 1};
    return run_clip(n, types, counts, grads, outs, a, (hipStream_t)stream);
}

int amulet_grad_norm_clip(int64_t n, const int32_t *types, const int64_t *counts, const void *const *grads, void *const *outs, float max_norm,
                          float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_tensors(n, types, counts, grads, outs);
    if (rc != AMULET_OK) return rc;
    if (!(max_norm >= 0.0f)) return AMULET_ERR_RANGE;
    if (!norm) return AMULET_ERR_NULL;
    rc = check_workspace(n, workspace, workspace_bytes);
    if (rc != AMULET_OK) return rc;
    note_kernel("grad_norm_clip", n);
    hipStream_t s = (hipStream_t)stream;
    const int64_t made = run_sums(n, types, counts, grads, (double *)workspace, s);
    if (made < 0) return (int)made;
    NormArgs a = {(double *)workspace, (int)made, norm, max_norm, 0};
    if (made > NORM_JOINED * NORM_BLOCKS) {   // (too many for every workgroup to add up)
        rc = launch_status(launch_norm_join(a, s));
        if (rc != AMULET_OK) return rc;
        a.given = 1;
    }
    return run_clip(n, types, counts, grads, outs, a, s);
}

}  // extern "C"
