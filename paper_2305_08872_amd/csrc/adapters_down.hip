// T[i] = scale[a(i)] X[i] A[a(i)]: a batch's rows, each by the first matrix of its adapter, M x r in fp32.
//
// Bound by X's bytes (many rows) or the adapters' (few).  A workgroup has up to BM rows of one segment and BN ranks; its waves share
// k, each with a ring of stages of its own in LDS (experts_tile.h), where all of it is read once from memory, and their
// sums are joined in the waves' order.  us, bf16, out of the caches: 16384 x 4096 by rank 16 29 (4.7 TB/s), 8192 x 4096 by rank 64 of 24 segments 25, a wave's
// way through its 64 stages, of which four are on their way.  (Fragments straight from memory instead, without LDS: neighbouring lanes of a matrix operand have rows
// of their own, a cache line for every 16 bytes, and 8192 x 4096 by rank 64 took 48 us.)
#include "adapters_segments.h"

namespace amulet {

// The rows are cut at every BM-th and where a segment begins.  Cut `k` of these (in order; at one row the segments' first), up to the
// next one: rows p0 .. p1 - 1 of segment s, or of none.
template <int BM>
__device__ __forceinline__ void rows_of_cut(const Segments &g, int k, int lane, int &p0, int &p1, int &s)
{
    if (g.S == 0) {   // (there need be no offsets)
        p0 = k < (g.M + BM - 1) / BM ? k * BM : g.M;
        p1 = p0 < g.M - BM ? p0 + BM : g.M;
        s = -1;
        return;
    }
    // place of segment x's beginning among all cuts: x and the tiles that begin before it
    auto place = [&](int64_t x) { return x + (clamp_row(g.offsets[x], g.M) + BM - 1) / BM; };
    int at = 0;   // how many segments that begin at cut k or before: 0 .. S + 1 (the last is the end of them all)
    for (int range = g.S + 1; range > 0;) {
        const int step = (range + 63) / 64;
        const int64_t x = at + (int64_t)lane * step;   // (known: those below `at`)
        const uint64_t before = __ballot(x <= g.S && place(x <= g.S ? x : g.S) <= k);
        const int n = __popcll(before);
        if (step == 1) { at += n; break; }
        if (n == 0) break;
        at += (n - 1) * step + 1;
        range = step - 1;
    }
    if (at > g.S + 1) at = g.S + 1;
    const int tile = k + 1 - at;   // tiles that begin there or before
    p0 = tile > 0 ? (tile - 1) * BM : 0;
    p1 = tile < (g.M + BM - 1) / BM ? tile * BM : g.M;
    if (at > 0) { const int x = clamp_row(g.offsets[at - 1], g.M); p0 = x > p0 ? x : p0; }
    if (at <= g.S) { const int x = clamp_row(g.offsets[at], g.M); p1 = x < p1 ? x : p1; }
    if (tile < 0 || p1 - p0 > BM) p1 = p0;   // (offsets that do not ascend)
    s = at - 1;
}

template <class T>
__global__ void __launch_bounds__(T::NT) adapters_down_kernel(const DownArgs a)
{
    static_assert(!T::AKS, "k lies along X's rows");
    static_assert(T::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kg = w / T::NW, wave = w % T::NW;
    const int wm = wave / T::WN * (T::BM / T::WM), wn = wave % T::WN * (T::BN / T::WN);   // the wave's first row and rank of the tile
    int p0, p1, s, lo, hi, g;
    rows_of_cut<T::BM>(a.rows, (int)blockIdx.x, lane, p0, p1, s);
    p0 = __builtin_amdgcn_readfirstlane(p0);
    p1 = __builtin_amdgcn_readfirstlane(p1);
    if (p0 >= p1) return;
    segment_rows(a.rows, __builtin_amdgcn_readfirstlane(s), lo, hi, g);
    g = __builtin_amdgcn_readfirstlane(g);
    const int from = (int)blockIdx.y * T::BN, r0 = T::BKS ? inside(from, T::BN, a.r) : from;
    const int K = g < 0 ? 0 : a.K;

    xt_f4 acc[T::MI][T::NI];
    auto same = [](int i) { return i; };
    Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> sa = {};
    Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> sb = {};
    if (K > 0) {
        const char *const A = (const char *)a.A + (int64_t)g * a.group_a * 2;
        sa.start_kc((const char *)a.X, a.ldx * 2, p0, p1, K, kg * T::BK, wave, lane, same, true);
        if constexpr (T::BKS) sb.start_ks(A, a.lda * 2, nullptr, 0, r0, a.r, K, kg * T::BK, wave, lane);
        else sb.start_kc(A, a.lda * 2, r0, a.r, K, kg * T::BK, wave, lane, same, true);
    }
    if (!tile_sums<T>(sa, sb, 0, K, wave, kg, lane, same, TileScales(), false, acc)) return;
    const float scale = g >= 0 && a.scales ? a.scales[g] : 1.0f;
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] *= scale;   // (zeros stay zeros: a scale of no adapter is 1)
    store_sums<T>(acc, a.T, EXPERTS_FP32, lane, r0 + wn, from, a.r, [&](int mi) -> int64_t {
        const int i = p0 + wm + mi * 16 + (lane & 15);
        return i < p1 ? (int64_t)i * a.ldt : -1;
    });
}

// (a dimension of a grid holds 2^32 - 1 work-items)
static bool fits(int64_t cuts, int threads) { return cuts <= 0xffffffffLL / threads; }

template <class T>
static hipError_t launch_tile(const DownArgs &a, hipStream_t s)
{
    const int64_t cuts = ((int64_t)a.rows.M + T::BM - 1) / T::BM + a.rows.S + 1;
    if (!fits(cuts, T::NT)) return hipErrorInvalidConfiguration;
    static const hipError_t granted = hipFuncSetAttribute((const void *)adapters_down_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
    adapters_down_kernel<T><<<dim3((unsigned)cuts, (unsigned)((a.r + T::BN - 1) / T::BN)), dim3(T::NT), T::LDS, s>>>(a);
    return hipGetLastError();
}
template <int ELEM, bool KS>
static hipError_t launch_down(const DownArgs &a, hipStream_t s)
{
    // Rows to a workgroup: a block where segments are shorter; 32, or 64 where those would be more than one to a compute unit (an adapter's matrix is
    // read once for as many).  us, 32 / 64 rows, rank 64, out of the caches: 8192 x 4096 of one segment 21 / 25, of 24 segments 39 / 26, 2048 x
    // 4096 13 / 15.  Blocks too, four workgroups to a compute unit, where up to 32 ranks have more than a round of 64 rows, whose last ones would
    // be alone: 16384 x 4096 rank 16 31 / 42 us, 65536 x 4096 99 / 116, 16384 x 4096 rank 32 38 / 43.
    const int64_t M = a.rows.M, S = a.rows.S, ranks = a.r <= 16 ? 16 : a.r <= 32 ? 32 : 64;
    const bool rounds = M / 64 + S > compute_units(), held = fits(M / 16 + S + 2, 256);
    const int rows = M < 16 * S ? 16 : (M / 32 + S) * ((a.r + ranks - 1) / ranks) <= compute_units() ? 32 : rounds && a.r <= 32 && held ? 16 : 64;
    if (a.r <= 16)
        return rows == 16 && rounds ? launch_tile<ExpertTile<ELEM, 16, 16, 1, 1, 4, 3, false, KS>>(a, s)
               : rows == 16 ? launch_tile<ExpertTile<ELEM, 16, 16, 1, 1, 8, 4, false, KS>>(a, s)
               : rows == 32 ? launch_tile<ExpertTile<ELEM, 32, 16, 1, 1, 8, 3, false, KS>>(a, s) : launch_tile<ExpertTile<ELEM, 64, 16, 1, 1, 4, 3, false, KS>>(a, s);
    if (a.r <= 32)
        return rows == 16 && rounds ? launch_tile<ExpertTile<ELEM, 16, 32, 1, 1, 4, 3, false, KS>>(a, s)
               : rows == 16 ? launch_tile<ExpertTile<ELEM, 16, 32, 1, 1, 8, 3, false, KS>>(a, s)
               : rows == 32 ? launch_tile<ExpertTile<ELEM, 32, 32, 1, 1, 4, 4, false, KS>>(a, s) : launch_tile<ExpertTile<ELEM, 64, 32, 1, 1, 4, 3, false, KS>>(a, s);
    return rows == 16 ? launch_tile<ExpertTile<ELEM, 16, 64, 1, 1, 4, 3, false, KS>>(a, s)
           : rows == 32 ? launch_tile<ExpertTile<ELEM, 32, 64, 1, 1, 4, 3, false, KS>>(a, s) : launch_tile<ExpertTile<ELEM, 64, 64, 2, 2, 1, 5, false, KS>>(a, s);
}

hipError_t launch_adapters_down(int type, const DownArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    if (type == EXPERTS_BF16) return a.across ? launch_down<EXPERTS_BF16, true>(a, s) : launch_down<EXPERTS_BF16, false>(a, s);
    return a.across ? launch_down<EXPERTS_FP16, true>(a, s) : launch_down<EXPERTS_FP16, false>(a, s);
}

}  // namespace amulet
