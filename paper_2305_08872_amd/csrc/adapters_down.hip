// T[i] = scale[a(i)] X[i] A[a(i)]: a batch's rows, each by the first matrix of its adapter, M x r in fp32.
//
// Bound by X's bytes (many rows) or the adapters' (few).  A workgroup has up to 16 MI rows of one segment and 16 RI ranks, and its
// eight waves share k: each takes a line of 128 bytes of every eighth, all of X's and A's fragments straight from memory into the matrix
// instruction, and the sums are joined in LDS in the waves' order.
#include "adapters_segments.h"

namespace amulet {

constexpr int kDownWaves = 8;

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

template <int ELEM, int MI, int RI, bool ACROSS>
__global__ void __launch_bounds__(64 * kDownWaves) adapters_down_kernel(const DownArgs a)
{
    constexpr int BM = 16 * MI, BK = 64;
    __shared__ xt_f4 sums[kDownWaves][MI * RI][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int p0, p1, s;
    rows_of_cut<BM>(a.rows, (int)blockIdx.x, lane, p0, p1, s);
    p0 = __builtin_amdgcn_readfirstlane(p0);
    p1 = __builtin_amdgcn_readfirstlane(p1);
    if (p0 >= p1) return;
    int lo, hi, g;
    segment_rows(a.rows, __builtin_amdgcn_readfirstlane(s), lo, hi, g);
    g = __builtin_amdgcn_readfirstlane(g);
    const int r0 = (int)blockIdx.y * 16 * RI, i = lane & 15, b = lane >> 4;

    xt_f4 acc[MI][RI];
#pragma unroll
    for (int m = 0; m < MI; ++m)
#pragma unroll
        for (int n = 0; n < RI; ++n) acc[m][n] = xt_f4{0, 0, 0, 0};
    if (g >= 0) {
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        const char *x[MI];
#pragma unroll
        for (int m = 0; m < MI; ++m) {
            const int row = p0 + m * 16 + i;
            x[m] = (const char *)a.X + (int64_t)(row < p1 ? row : p1 - 1) * a.ldx * 2;
        }
        const char *const base = (const char *)a.A + (int64_t)g * a.group_a * 2;
        const char *y[RI];
#pragma unroll
        for (int n = 0; n < RI; ++n) {
            const int c = r0 + n * 16 + i;
            const int64_t at = c < a.r ? c : a.r - 1;
            y[n] = base + (ACROSS ? at * 2 : at * a.lda * 2);
        }
        auto read_x = [&](int m, int k, bool whole) -> xt_u4 {   // 8 k from k on
            if (whole) return __builtin_bit_cast(xt_u4, *(const u4 *)(x[m] + k * 2));
            return k < a.K ? load_unit<2>(x[m], k * 2, a.K * 2) : xt_u4{0, 0, 0, 0};
        };
        auto read_a = [&](int n, int k, bool whole) -> xt_u4 {
            if constexpr (!ACROSS) {
                if (whole) return __builtin_bit_cast(xt_u4, *(const u4 *)(y[n] + k * 2));
                return k < a.K ? load_unit<2>(y[n], k * 2, a.K * 2) : xt_u4{0, 0, 0, 0};
            } else {
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = whole || k + j < a.K ? *(const uint16_t *)(y[n] + (int64_t)(k + j) * a.lda * 2) : 0u;
                return xt_u4{v[0] | (v[1] << 16), v[2] | (v[3] << 16), v[4] | (v[5] << 16), v[6] | (v[7] << 16)};
            }
        };
        auto line = [&](int k0, bool whole) {
            xt_u4 fx[2][MI], fa[2][RI];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 32 * h + 8 * b;
#pragma unroll
                for (int m = 0; m < MI; ++m) fx[h][m] = read_x(m, k, whole);
#pragma unroll
                for (int n = 0; n < RI; ++n) fa[h][n] = read_a(n, k, whole);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < MI; ++m)
#pragma unroll
                    for (int n = 0; n < RI; ++n) acc[m][n] = mma16<ELEM>(fa[h][n], fx[h][m], acc[m][n]);
        };
        int k0 = wave * BK;
        for (; k0 + BK <= a.K; k0 += kDownWaves * BK) line(k0, true);
        if (k0 < a.K) line(k0, false);
    }
#pragma unroll
    for (int m = 0; m < MI; ++m)
#pragma unroll
        for (int n = 0; n < RI; ++n) sums[wave][m * RI + n][lane] = acc[m][n];
    __syncthreads();
    const float scale = g >= 0 && a.scales ? a.scales[g] : 1.0f;
    for (int f = wave; f < MI * RI; f += kDownWaves) {
        xt_f4 t = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w) t += sums[w][f][lane];
        const int row = p0 + f / RI * 16 + i, c = r0 + f % RI * 16 + 4 * b;
        const float v[4] = {g < 0 ? 0.0f : t[0] * scale, g < 0 ? 0.0f : t[1] * scale, g < 0 ? 0.0f : t[2] * scale, g < 0 ? 0.0f : t[3] * scale};
        if (row < p1) store_out<4>(a.T, EXPERTS_FP32, (int64_t)row * a.ldt, c, 0, a.r, v);
    }
}

template <int ELEM, int MI, int RI>
static hipError_t launch_down(const DownArgs &a, hipStream_t s)
{
    const int64_t cuts = ((int64_t)a.rows.M + 16 * MI - 1) / (16 * MI) + a.rows.S + 1;
    const dim3 grid((unsigned)cuts, (unsigned)((a.r + 16 * RI - 1) / (16 * RI)));
    if (a.across) adapters_down_kernel<ELEM, MI, RI, true><<<grid, dim3(64 * kDownWaves), 0, s>>>(a);
    else adapters_down_kernel<ELEM, MI, RI, false><<<grid, dim3(64 * kDownWaves), 0, s>>>(a);
    return hipGetLastError();
}
template <int ELEM>
static hipError_t launch_down(const DownArgs &a, hipStream_t s)
{
    const bool few = a.rows.M < 16 * (int64_t)a.rows.S;
    if (a.r <= 16) return few ? launch_down<ELEM, 1, 1>(a, s) : launch_down<ELEM, 2, 1>(a, s);
    if (a.r <= 32) return few ? launch_down<ELEM, 1, 2>(a, s) : launch_down<ELEM, 2, 2>(a, s);
    return few ? launch_down<ELEM, 1, 4>(a, s) : launch_down<ELEM, 2, 4>(a, s);
}

hipError_t launch_adapters_down(int type, const DownArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    return type == EXPERTS_BF16 ? launch_down<EXPERTS_BF16>(a, s) : launch_down<EXPERTS_FP16>(a, s);
}

}  // namespace amulet
