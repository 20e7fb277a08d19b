// R[i] = X[i] W + T[i] B[a(i)]: the products by rows of one shared matrix (experts_tile.h), whose sums begin with the adapters'.
//
// A wave finds the segments that its rows meet and adds T B of each, straight from memory into the matrix instruction, while the
// first stages of X and W are on their way.  T is fp32 and stays so: as two bf16 pieces where R has 16 bits (a rounding of 2^-17 to
// each value, under R's of 2^-9 or 2^-12), as three, exactly, where it has 32; B of fp16 as two, exactly (fp16 products would be the
// shorter way, but T may lie outside its range).  Pieces and ranks lie one behind the other along the instruction's k: a rank of 16
// in two pieces fills it.  An instruction's sums are taken over by the lanes whose row is the segment's.
#ifndef AMULET_ADAPTERS_UP_IMPL_H
#define AMULET_ADAPTERS_UP_IMPL_H

#include "adapters_segments.h"

namespace amulet {

template <class T>
struct AddAdapters {
    // (segment, k step) pairs whose operands are on their way at a time
    static constexpr int PAIRS = T::MI <= 1 ? 4 : T::MI <= 2 && T::NI <= 2 ? 2 : 1;
    // row blocks whose values of T are: the larger tiles have no registers for all
    static constexpr int ROWS = T::MI < 2 ? T::MI : 2;
    const UpArgs &a;
    int row0, col0, lane, kg;   // the wave's first row and column

    struct Pair {
        int adapter, lo, hi, step;
    };

    // the lane's 8 ranks (from `unit` * 8 on) of column n of an adapter's matrix; zeros past the rank
    __device__ __forceinline__ xt_u4 read_b(const char *b, int n, int unit, bool there) const
    {
        xt_u4 v = {0, 0, 0, 0};
        if (!a.across) {
            const char *const row = b + (int64_t)n * a.ldb * 2;
            if (there) v = load_unit<2>(row, unit * 16, a.r * 2);
        } else {
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = unit * 8 + j;
                x[j] = there && k < a.r ? *(const uint16_t *)(b + ((int64_t)k * a.ldb + n) * 2) : 0u;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = x[2 * j] | (x[2 * j + 1] << 16);
        }
        return v;
    }
    __device__ __forceinline__ void read_t(int row, int unit, bool there, float (&t)[8]) const
    {
        const float *const p = a.T + (int64_t)row * a.ldt + unit * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = there && unit * 8 + j < a.r ? p[j] : 0.0f;
    }

    __device__ __forceinline__ void operator()(xt_f4 (&acc)[T::MI][T::NI]) const
    {
        if (a.r == 0 || a.rows.S == 0) return;
        const int row1 = row0 + T::MI * 16 < a.rows.M ? row0 + T::MI * 16 : a.rows.M;
        const int i = lane & 15, b = lane >> 4;
        const int pieces = a.mm.out == EXPERTS_FP32 ? 3 : 2, of_b = T::ELEM == EXPERTS_FP16 ? 2 : 1;
        const int units = (a.r + 7) / 8, ways = pieces * of_b, steps = (units * ways + 3) / 4;

        int chunk = segment_of(a.rows, row0, lane);
        int lo, hi, adapter;
        uint64_t left;
        bool more;
        auto look = [&]() {   // the segments from `chunk` on that the rows meet
            segment_rows(a.rows, chunk + lane, lo, hi, adapter);
            left = __ballot(adapter >= 0 && hi > lo && lo < row1 && hi > row0);
            more = chunk + 64 < a.rows.S && !__ballot(chunk + lane < a.rows.S && lo >= row1);
        };
        look();
        int step = 0, met = 0;
        auto next = [&](Pair &p) -> bool {
            for (;;) {
                if (left == 0) {
                    if (!more) return false;
                    chunk += 64;
                    look();
                    continue;
                }
                if (T::WK > 1 && met % T::WK != kg) {   // (the k groups take the segments in turn)
                    left &= left - 1;
                    ++met;
                    continue;
                }
                const int l = __builtin_ctzll(left);
                p = {__builtin_amdgcn_readlane(adapter, l), __builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l), step};
                if (++step == steps) { step = 0; left &= left - 1; ++met; }
                return true;
            }
        };
        for (;;) {
            Pair p[PAIRS];
            xt_u4 vb[PAIRS][T::NI];
            int n = 0;
            for_each<PAIRS>([&](auto which) {
                constexpr int q = decltype(which)::value;
                if (n < q || !next(p[q])) return;
                n = q + 1;
                const int at = 4 * p[q].step + b, way = at / units, unit = at - way * units;
                const char *const m = (const char *)a.B + (int64_t)p[q].adapter * a.group_b * 2;
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) {
                    const int c = col0 + (T::PERM ? (ni >> 1) * 32 + 8 * (i >> 2) + (i & 3) + (ni & 1) * 4 : ni * 16 + i);
                    vb[q][ni] = read_b(m, c < a.mm.N ? c : a.mm.N - 1, unit, at < units * ways);
                }
            });
            if (n == 0) break;
#pragma unroll
            for (int m0 = 0; m0 < T::MI; m0 += ROWS) {
                float vt[PAIRS][ROWS][8];
                auto meets = [&](int q, int m) { return q < n && row0 + (m0 + m) * 16 < p[q].hi && row0 + (m0 + m) * 16 + 16 > p[q].lo; };
#pragma unroll
                for (int q = 0; q < PAIRS; ++q)
#pragma unroll
                    for (int m = 0; m < ROWS; ++m)
                        if (meets(q, m)) {
                            const int at = 4 * p[q].step + b, row = row0 + (m0 + m) * 16 + i;
                            read_t(row < a.rows.M ? row : a.rows.M - 1, at % units, at < units * ways, vt[q][m]);
                        }
#pragma unroll
                for (int q = 0; q < PAIRS; ++q) {
                    if (q >= n) continue;
                    const int way = (4 * p[q].step + b) / units, of_t = way / of_b;
                    if constexpr (T::ELEM == EXPERTS_FP16)
                        if (m0 == 0)
#pragma unroll
                            for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    vb[q][ni][j] = bf16_pair(piece_of(half_of<EXPERTS_FP16>(vb[q][ni][j], 0), way % 2, 2), piece_of(half_of<EXPERTS_FP16>(vb[q][ni][j], 1), way % 2, 2));
#pragma unroll
                    for (int m = 0; m < ROWS; ++m) {
                        if (!meets(q, m)) continue;
                        const int row = row0 + (m0 + m) * 16 + i;
                        xt_u4 t;
#pragma unroll
                        for (int j = 0; j < 4; ++j) t[j] = bf16_pair(piece_of(vt[q][m][2 * j], of_t, pieces), piece_of(vt[q][m][2 * j + 1], of_t, pieces));
                        const bool in = row >= p[q].lo && row < p[q].hi;
#pragma unroll
                        for (int ni = 0; ni < T::NI; ++ni) {
                            const xt_f4 x = mma16<EXPERTS_BF16>(vb[q][ni], t, acc[m0 + m][ni]);
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[m0 + m][ni][v] = in ? x[v] : acc[m0 + m][ni][v];
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (n < PAIRS) break;
        }
    }
};

template <class T>
__global__ void __launch_bounds__(T::NT) __attribute__((amdgpu_waves_per_eu(2))) adapters_up_kernel(const UpArgs u)
{
    static_assert(!T::AKS && !T::FP8, "16-bit products by rows");
    static_assert(T::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
    const ExpertsArgs &a = u.mm;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kg = w / T::NW, wave = w % T::NW;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    RowTile t;
    if (!find_row_tile<T::BM>(a, tiles_n, blockIdx.x, t)) return;
    const int row0 = t.tm * T::BM, from = t.tn * T::BN;
    const int col0 = T::BKS ? inside(from, T::BN, a.N) : from;
    const int wm = wave / T::WN, wn = wave % T::WN;
    const int wave_row = row0 + wm * (T::BM / T::WM), wave_col = col0 + wn * (T::BN / T::WN);
    xt_f4 acc[T::MI][T::NI];
    auto a_row = [](int i) { return i; };
    Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> sa = {};
    Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> sb = {};
    if (a.K > 0) {
        sa.start_kc((const char *)a.A, a.lda * T::ES, row0, a.M, a.K, kg * T::BK, wave, lane, a_row, true);
        if constexpr (T::BKS) sb.start_ks((const char *)a.B, a.ldb * T::ES, nullptr, 0, col0, a.N, a.K, kg * T::BK, wave, lane);
        else sb.start_kc((const char *)a.B, a.ldb * T::ES, col0, a.N, a.K, kg * T::BK, wave, lane, a_row, true);
    }
    const AddAdapters<T> adapters = {u, wave_row, wave_col, lane, kg};
    const bool idle = wave_row >= a.M;
    if constexpr (T::BM >= 256) {   // (beside its stages' state it has no registers for them: at the end)
        tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc);
        if (!idle) adapters(acc);
    } else if (!tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc, adapters)) return;
    store_sums<T>(acc, a.R, a.out, lane, wave_col, from, a.N, [&](int mi) -> int64_t {
        const int i = wave_row + mi * 16 + (lane & 15);
        return i < a.M ? (int64_t)i * a.ldr : -1;
    });
}

template <class T>
inline hipError_t launch_adapters_tile(const UpArgs &a, int64_t blocks, hipStream_t s)
{
    if (blocks <= 0) return hipSuccess;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    static const hipError_t granted = hipFuncSetAttribute((const void *)adapters_up_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
    adapters_up_kernel<T><<<dim3((unsigned)blocks), dim3(T::NT), T::LDS, s>>>(a);
    return hipGetLastError();
}

template <int ELEM, bool BKS>
inline hipError_t launch_adapters_layout(int tile, const UpArgs &a, int64_t blocks, hipStream_t s)
{
    switch (tile) {
    case EXPERTS_256x256: return launch_adapters_tile<ExpertTile<ELEM, 256, 256, 2, 4, 1, 2, false, BKS>>(a, blocks, s);
    case EXPERTS_128x128: return launch_adapters_tile<ExpertTile<ELEM, 128, 128, 2, 2, 1, 2, false, BKS>>(a, blocks, s);
    case EXPERTS_64x128: return launch_adapters_tile<ExpertTile<ELEM, 64, 128, 2, 2, 1, 3, false, BKS>>(a, blocks, s);
    case EXPERTS_64x64: return launch_adapters_tile<ExpertTile<ELEM, 64, 64, 2, 2, 1, 3, false, BKS>>(a, blocks, s);
    case EXPERTS_64x64_K2: return launch_adapters_tile<ExpertTile<ELEM, 64, 64, 2, 2, 2, 3, false, BKS>>(a, blocks, s);
    default: return launch_adapters_tile<ExpertTile<ELEM, 16, 32, 1, 1, 4, 3, false, BKS>>(a, blocks, s);
    }
}

template <int ELEM>
inline hipError_t launch_adapters_up(int tile, bool w_across, const UpArgs &a, int64_t blocks, hipStream_t s)
{
    return w_across ? launch_adapters_layout<ELEM, true>(tile, a, blocks, s) : launch_adapters_layout<ELEM, false>(tile, a, blocks, s);
}

}  // namespace amulet
#endif
