// R[i] = X[i] W + T[i] B[a(i)]: the products by rows of one shared matrix (experts_tile.h), to whose sums the adapters' are added.
//
// T is fp32 and stays so: it enters as two bf16 pieces where R has 16 bits (a rounding of 2^-15 to each value at most, under R's of 2^-8 or
// 2^-11), as three, exactly, where it has 32; B of fp16 as two, exactly (fp16 products would be the shorter way, but T may lie
// outside its range).  A workgroup lays the pieces of its rows out in LDS.  A block of 16 rows that a segment has in part takes an
// instruction's sums over in the lanes whose row it is: nothing of another segment's operands is seen, not even an infinity times zero.
//
// Tiles whose k is shared by groups of waves (few rows: a decoding batch, many short segments) add the adapters while the first stages of X
// and W are on their way: each wave takes B of eight segments at a time from memory straight into the matrix instruction.  The
// others do it when their own sums are done and the stages' LDS is free: B of as many segments as it holds is laid out beside T.
#ifndef AMULET_ADAPTERS_UP_IMPL_H
#define AMULET_ADAPTERS_UP_IMPL_H

#include "adapters_segments.h"

namespace amulet {

// Units: 8 ranks, of which an instruction has four.  Ways: the pieces of T times those of B.
struct Ways {
    int units, ways;
    bool packed;   // few units: an instruction's four groups of lanes have ways too, one behind the other
    __device__ __forceinline__ Ways(int n, int w) : units(n), ways(w), packed(n <= 2) {}
    __device__ __forceinline__ int steps() const { return packed ? (units * ways + 3) / 4 : (units + 3) / 4 * ways; }
    // of step s, in the lanes of group b: unit and way; whether there is one
    __device__ __forceinline__ bool at(int s, int b, int &unit, int &way) const
    {
        if (packed) {
            const int x = 4 * s + b;
            unit = units == 1 ? 0 : x & 1;
            way = units == 1 ? x : x >> 1;
        } else {
            const int q = s / ways;
            unit = 4 * q + b;
            way = s - q * ways;
        }
        return unit < units && way < ways;
    }
};

// What both ways of adding the adapters share
template <class T>
struct Adapters {
    static constexpr int OF_B = T::ELEM == EXPERTS_FP16 ? 2 : 1;   // pieces of a value of B
    const UpArgs &a;
    int tile_row, tile_col, row0, col0, lane, kg;   // the tile's first row and column, the wave's
    bool idle;

    // 8 ranks (from `unit` * 8 on) of column n of an adapter's matrix; zeros past the rank
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
    // one of its pieces
    static __device__ __forceinline__ xt_u4 piece_of_b(xt_u4 v, int which)
    {
        if constexpr (OF_B > 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = bf16_pair(piece_of(half_of<EXPERTS_FP16>(v[j], 0), which, 2), piece_of(half_of<EXPERTS_FP16>(v[j], 1), which, 2));
        return v;
    }
    // T of the tile's rows, units u0 .. u0 + n - 1, as pieces: slot (unit * pieces + piece) has 16 bytes of every row
    __device__ __forceinline__ void lay_out_t(char *lds, int u0, int n, int pieces) const
    {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        for (int at = (int)threadIdx.x; at < n * T::BM; at += T::NT) {
            const int line = at / n, unit = at - line * n, row = tile_row + line, k = (u0 + unit) * 8;
            float t[8];
            const float *const p = a.T + (int64_t)row * a.ldt + k;
            if (row < a.rows.M && k + 8 <= a.r) {
                const f4 x = *(const f4 *)p, y = *(const f4 *)(p + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { t[j] = x[j]; t[4 + j] = y[j]; }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = row < a.rows.M && k + j < a.r ? p[j] : 0.0f;
            }
            for (int piece = 0; piece < pieces; ++piece) {
                xt_u4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = bf16_pair(piece_of(t[2 * j], piece, pieces), piece_of(t[2 * j + 1], piece, pieces));
                *(xt_u4 *)(lds + ((unit * pieces + piece) * T::BM + line) * 16) = v;
            }
        }
    }
    // an instruction's products added to block m, in the rows lo .. hi - 1
    template <int mi>
    __device__ __forceinline__ void add_block(xt_f4 (&acc)[T::MI][T::NI], const char *t_at, bool there, int lo, int hi, const xt_u4 (&vb)[T::NI]) const
    {
        const int first = row0 + mi * 16, row = first + (lane & 15);
        if (!(first < hi && first + 16 > lo)) return;
        xt_u4 t = *(const xt_u4 *)(t_at + mi * 256);
        if (!there) t = xt_u4{0, 0, 0, 0};
        const bool in = row >= lo && row < hi;
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) {
            const xt_f4 x = mma16<EXPERTS_BF16>(vb[ni], t, acc[mi][ni]);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[mi][ni][v] = in ? x[v] : acc[mi][ni][v];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // a lane's column of fragment ni, of the wave's
    static __device__ __forceinline__ int column(int ni, int lane)
    {
        const int i = lane & 15;
        return T::PERM ? (ni >> 1) * 32 + 8 * (i >> 2) + (i & 3) + (ni & 1) * 4 : ni * 16 + i;
    }
};

// The segments that rows first .. last - 1 meet, 64 at a time: their rows and adapters in the lanes
struct Meeting {
    int chunk, lo, hi, adapter;
    uint64_t which;
    bool more;
    __device__ __forceinline__ void start(const Segments &g, int first, int last, int lane)
    {
        chunk = segment_of(g, first, lane);
        look(g, first, last, lane);
    }
    __device__ __forceinline__ void look(const Segments &g, int first, int last, int lane)
    {
        segment_rows(g, chunk + lane, lo, hi, adapter);
        which = __ballot(adapter >= 0 && hi > lo && lo < last && hi > first);
        more = chunk + 64 < g.S && !__ballot(chunk + lane < g.S && lo >= last);
    }
    __device__ __forceinline__ void next(const Segments &g, int first, int last, int lane) { chunk += 64; look(g, first, last, lane); }
};

// From memory: (segment, step) pairs, PAIRS of them on their way at a time; the k groups take the segments in turn
template <class T>
struct AddFromMemory : Adapters<T> {
    static constexpr int ROOM = T::BM >= 64 ? 32 * 1024 : 8 * 1024;   // for T, beside the ring
    static constexpr int LDS = T::LDS + ROOM, SLOTS = ROOM / (T::BM * 16);
    static constexpr int PAIRS = 8 / Adapters<T>::OF_B;
    static_assert(SLOTS >= 3, "one unit in three pieces");
    __device__ __forceinline__ AddFromMemory(const Adapters<T> &x) : Adapters<T>(x) {}

    struct Pair {
        int adapter, lo, hi, step;
    };
    __device__ __forceinline__ void operator()(xt_f4 (&acc)[T::MI][T::NI]) const
    {
        const UpArgs &a = this->a;
        if (a.r == 0 || a.rows.S == 0) return;
        char *const lds = xt_smem + T::LDS;
        const int pieces = a.mm.out == EXPERTS_FP32 ? 3 : 2, units = (a.r + 7) / 8, most = SLOTS / pieces;
        for (int u0 = 0; u0 < units; u0 += most) {
            const int n = units - u0 < most ? units - u0 : most;
            if (u0 > 0) __syncthreads();
            this->lay_out_t(lds, u0, n, pieces);
            meet<T::NW * T::WK>();
            if (!this->idle) add(acc, lds, u0, n, pieces);
        }
    }
    __device__ __forceinline__ void add(xt_f4 (&acc)[T::MI][T::NI], const char *lds, int u0, int n_units, int pieces) const
    {
        const UpArgs &a = this->a;
        const int lane = this->lane, row0 = this->row0, b = lane >> 4, row1 = row0 + T::MI * 16 < a.rows.M ? row0 + T::MI * 16 : a.rows.M;
        const Ways ways(n_units, pieces * this->OF_B);
        const int steps = ways.steps();
        Meeting m;
        m.start(a.rows, row0, row1, lane);
        int step = 0, met = 0;
        auto next = [&](Pair &p) -> bool {
            for (;;) {
                if (m.which == 0) {
                    if (!m.more) return false;
                    m.next(a.rows, row0, row1, lane);
                    continue;
                }
                if (met % T::WK != this->kg) {
                    m.which &= m.which - 1;
                    ++met;
                    continue;
                }
                const int l = __builtin_ctzll(m.which);
                p = {__builtin_amdgcn_readlane(m.adapter, l), __builtin_amdgcn_readlane(m.lo, l), __builtin_amdgcn_readlane(m.hi, l), step};
                if (++step == steps) { step = 0; m.which &= m.which - 1; ++met; }
                return true;
            }
        };
        const char *const t_row = lds + (row0 - this->tile_row + (lane & 15)) * 16;
        for (;;) {
            Pair p[PAIRS];
            xt_u4 vb[PAIRS][T::NI];
            int n = 0;
            for_each<PAIRS>([&](auto which) {
                constexpr int q = decltype(which)::value;
                if (n < q || !next(p[q])) return;
                n = q + 1;
                int unit, way;
                const bool there = ways.at(p[q].step, b, unit, way);
                const char *const from = (const char *)a.B + (int64_t)p[q].adapter * a.group_b * 2;
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) {
                    const int c = this->col0 + this->column(ni, lane);
                    vb[q][ni] = this->read_b(from, c < a.mm.N ? c : a.mm.N - 1, u0 + unit, there);
                }
            });
            if (n == 0) break;
            for_each<PAIRS>([&](auto which) {
                constexpr int q = decltype(which)::value;
                if (q >= n) return;
                int unit, way;
                const bool there = ways.at(p[q].step, b, unit, way);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) vb[q][ni] = this->piece_of_b(vb[q][ni], way % this->OF_B);
                const char *const t_at = t_row + (there ? unit * pieces + way / this->OF_B : 0) * (T::BM * 16);
                for_each<T::MI>([&](auto mi) { this->template add_block<decltype(mi)::value>(acc, t_at, there, p[q].lo, p[q].hi, vb[q]); });
            });
            if (n < PAIRS) break;
        }
    }
};

// Through LDS: T's pieces and B's (slot (unit * pieces + piece) of a segment has 16 bytes of every column)
template <class T>
struct AddFromLds : Adapters<T> {
    static constexpr int LDS = T::LDS, ROOM = T::S * T::STAGE - 1024;   // (a list of 64 segments behind it)
    static constexpr int OF_B = Adapters<T>::OF_B;
    __device__ __forceinline__ AddFromLds(const Adapters<T> &x) : Adapters<T>(x) {}

    __device__ __forceinline__ void operator()(xt_f4 (&acc)[T::MI][T::NI]) const
    {
        const UpArgs &a = this->a;
        if (a.r == 0 || a.rows.S == 0) return;
        const int lane = this->lane, row0 = this->tile_row, row1 = row0 + T::BM < a.rows.M ? row0 + T::BM : a.rows.M;
        const int pieces = a.mm.out == EXPERTS_FP32 ? 3 : 2, units = (a.r + 7) / 8;
        const int t_unit = pieces * T::BM * 16, b_unit = OF_B * T::BN * 16;
        const int most = ROOM / (t_unit + b_unit);
        static_assert(ROOM >= (3 * T::BM + OF_B * T::BN) * 16, "a unit of both");
        int4 *const list = (int4 *)(xt_smem + ROOM);
        for (int u0 = 0; u0 < units; u0 += most) {
            const int n_units = units - u0 < most ? units - u0 : most;
            __syncthreads();   // (what lies there is read no more)
            this->lay_out_t(xt_smem, u0, n_units, pieces);
            char *const lds_b = xt_smem + n_units * t_unit;
            const int at_once = (ROOM - n_units * t_unit) / (n_units * b_unit);   // segments, one at least
            const Ways ways(n_units, pieces * OF_B);
            const int steps = ways.steps();
            Meeting m;
            m.start(a.rows, row0, row1, lane);
            for (;;) {
                const int met = __popcll(m.which);
                if (threadIdx.x < 64 && ((m.which >> lane) & 1))
                    list[__popcll(m.which & ((1ull << lane) - 1))] = int4{m.adapter, m.lo, m.hi, 0};
                for (int s0 = 0; s0 < met; s0 += at_once) {
                    const int n = met - s0 < at_once ? met - s0 : at_once;
                    __syncthreads();   // the list is there; B's slots are read no more
                    lay_out_b(lds_b, list + s0, n, u0, n_units);
                    __syncthreads();
                    if (!this->idle)
                        for (int k = 0; k < n; ++k) {
                            const int4 seg = list[s0 + k];
                            const int lo = __builtin_amdgcn_readfirstlane(seg.y), hi = __builtin_amdgcn_readfirstlane(seg.z);
                            if (lo < this->row0 + T::MI * 16 && hi > this->row0) products(acc, lds_b + k * n_units * b_unit, lo, hi, ways, steps, pieces);
                        }
                }
                if (!m.more) break;
                __syncthreads();       // (the list is read no more)
                m.next(a.rows, row0, row1, lane);
            }
        }
    }
    // B of n segments' adapters, units u0 .. u0 + units - 1, the tile's columns
    __device__ __forceinline__ void lay_out_b(char *lds, const int4 *list, int n, int u0, int units) const
    {
        const UpArgs &a = this->a;
        // neighbouring threads: neighbouring addresses
        const int fast = a.across ? T::BN : units, slow = a.across ? units : T::BN;
        for (int at = (int)threadIdx.x; at < n * units * T::BN; at += T::NT) {
            const int x = at / fast, f = at - x * fast, k = x / slow, y = x - k * slow;
            const int unit = a.across ? y : f, line = a.across ? f : y;
            const int c = this->tile_col + line;
            const xt_u4 v = this->read_b((const char *)a.B + (int64_t)list[k].x * a.group_b * 2, c < a.mm.N ? c : a.mm.N - 1, u0 + unit, true);
#pragma unroll
            for (int p = 0; p < OF_B; ++p) *(xt_u4 *)(lds + (((k * units + unit) * OF_B + p) * T::BN + line) * 16) = this->piece_of_b(v, p);
        }
    }
    __device__ __forceinline__ void products(xt_f4 (&acc)[T::MI][T::NI], const char *lds_b, int lo, int hi, const Ways &ways, int steps, int pieces) const
    {
        const int lane = this->lane, b = lane >> 4;
        const char *const t_row = xt_smem + (this->row0 - this->tile_row + (lane & 15)) * 16;
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
            int unit, way;
            const bool there = ways.at(s, b, unit, way);
            const char *const t_at = t_row + (there ? unit * pieces + way / OF_B : 0) * (T::BM * 16);
            const char *const b_at = lds_b + ((there ? unit * OF_B + way % OF_B : 0) * T::BN + this->col0 - this->tile_col) * 16;
            xt_u4 vb[T::NI];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                vb[ni] = *(const xt_u4 *)(b_at + this->column(ni, lane) * 16);
                if (!there) vb[ni] = xt_u4{0, 0, 0, 0};
            }
            for_each<T::MI>([&](auto mi) { this->template add_block<decltype(mi)::value>(acc, t_at, there, lo, hi, vb); });
        }
    }
};

template <class T>
using AddAdapters = std::conditional_t<(T::WK > 1), AddFromMemory<T>, AddFromLds<T>>;

template <class T>
__global__ void __launch_bounds__(T::NT) __attribute__((amdgpu_waves_per_eu(2))) adapters_up_kernel(const UpArgs u)
{
    static_assert(!T::AKS && !T::FP8, "16-bit products by rows");
    static_assert(AddAdapters<T>::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
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
    const bool idle = wave_row >= a.M;
    const AddAdapters<T> adapters(Adapters<T>{u, row0, col0, wave_row, wave_col, lane, kg, idle});
    if constexpr (T::WK > 1) {
        if (!tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc, adapters)) return;
    } else {
        tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc);
        adapters(acc);
    }
    store_sums<T>(acc, a.R, a.out, lane, wave_col, from, a.N, [&](int mi) -> int64_t {
        const int i = wave_row + mi * 16 + (lane & 15);
        return i < a.M ? (int64_t)i * a.ldr : -1;
    });
}

template <class T>
inline hipError_t launch_adapters_tile(const UpArgs &a, int64_t blocks, hipStream_t s)
{
    constexpr int lds = AddAdapters<T>::LDS;
    if (blocks <= 0) return hipSuccess;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    static const hipError_t granted = hipFuncSetAttribute((const void *)adapters_up_kernel<T>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
    adapters_up_kernel<T><<<dim3((unsigned)blocks), dim3(T::NT), lds, s>>>(a);
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
