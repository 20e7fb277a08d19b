// R[i] = X[i] W + T[i] B[a(i)]: the products by rows of one shared matrix (experts_tile.h), to whose sums the adapters' are added.
//
// T is fp32 and stays so: it enters the matrix instructions as three bf16 pieces, all of its 24 bits (two, 16 bits, would be 3 % faster with rank 64 and
// were seen in results of 16 bits where X W and T B cancel: up to 29 times as far off as sums of 32 bits are); B of fp16 as two, exactly (fp16
// products would be the shorter way, but T may lie outside its range).  So a row's sums have the same bits of T whichever way they are added.  A workgroup lays the pieces of its rows out in LDS.  A block of 16 rows that a segment has in part takes an
// instruction's sums over in the lanes whose row it is: nothing of another segment's operands is seen, not even an infinity times zero.
//
// That is for tiles of many rows, when their own sums are done and the stages' LDS is free: B of as many segments as it holds is laid out
// beside T.  Tiles of few rows (whose k is shared by groups of waves) and batches of short segments take T and B from memory, row by
// row, on the vector ALU, while the first stages of X and W are on their way.
//
// Bound by the shared product's operations (many rows) or W's bytes (few).  us, bf16, beside the same call without adapters: 8192 x 8192 x 4096 by
// 24 segments, rank 64 497 / 424, rank 16 451 / 426, rank 64 of fp16 562 / 444; 16384 x 4096 x 4096, rank 16 454 / 439; 4096 x 4096 x 2048 by 32 segments, rank 64, results
// of 32 bits 88 / 65; 8 x 4096 x 4096, a segment to a row, rank 16 10.4 / 9.2; 208 rows of 192 segments, rank 32 24 / 17.
#ifndef AMULET_ADAPTERS_UP_IMPL_H
#define AMULET_ADAPTERS_UP_IMPL_H

#include "adapters_segments.h"

namespace amulet {

// Units: 8 ranks, of which an instruction has four.  Ways: the pieces of T times those of B.  What is read of B at a time (up to four units) is
// taken by as many instructions as it has ways, or, with one or two units, as all of these fill, one behind the other.
struct Ways {
    int units, ways;
    bool packed;
    __device__ __forceinline__ Ways(int n, int w) : units(n), ways(w), packed(n <= 2) {}
    __device__ __forceinline__ int reads() const { return (units + 3) / 4; }
    __device__ __forceinline__ int of_read(int read) const { return units - 4 * read < 4 ? units - 4 * read : 4; }   // units
    __device__ __forceinline__ int each() const { return packed ? (units * ways + 3) / 4 : ways; }                   // instructions
    // of instruction e of a read, in the lanes of group b: unit and way; whether there is one
    __device__ __forceinline__ bool at(int read, int e, int b, int &unit, int &way) const
    {
        const int x = 4 * e + b;
        unit = !packed ? 4 * read + b : units == 1 ? 0 : x & 1;
        way = !packed ? e : units == 1 ? x : x >> 1;
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

    // 8 ranks (from `unit` * 8 on, the first there) of column n of an adapter's matrix; zeros past the rank
    __device__ __forceinline__ xt_u4 read_b(const char *b, int n, int unit) const
    {
        xt_u4 v = {0, 0, 0, 0};
        if (!a.across) {
            const char *const row = b + (int64_t)n * a.ldb * 2;
            typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
            if ((a.r & 7) == 0) v = __builtin_bit_cast(xt_u4, *(const u4 *)(row + unit * 16));
            else v = load_unit<2>(row, unit * 16, a.r * 2);
        } else {
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = unit * 8 + j;
                x[j] = *(const uint16_t *)(b + ((int64_t)(k < a.r ? k : a.r - 1) * a.ldb + n) * 2);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = unit * 8 + j < a.r ? x[j] : 0u;
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
    // In LDS (AddFromLds) a slot has a unit of every line, 16 bytes each.  Its lines are turned by the unit, so that lanes that write neighbouring units
    // of a line reach other banks (by no more than pairs of lines: a read's clocks take four lanes here and four there), and B's lie
    // as its fragments read them.  Counted conflicts of 8192 x 8192 x 4096 with rank 64: an eighth of what lines in order have.
    static __device__ __forceinline__ int turn(int unit) { return (unit << 1) & 15; }
    static __device__ __forceinline__ int line_of_b(int line) { return T::PERM ? (line & ~31) | (line & 4) << 2 | (line >> 1 & 12) | (line & 3) : line; }
    // T of the tile's rows, units u0 .. u0 + n - 1, as pieces: slot (unit * pieces + piece) has 16 bytes of every row.  A thread has two items (8
    // ranks of a row) on their way at a time; no branch around a read: what is not there is read at the edge and becomes zeros.
    static constexpr int T_ITEMS = 2;
    __device__ __forceinline__ void item_of_t(int at, int n, int &line, int &unit) const
    {
        line = at / n;
        unit = at - line * n;
    }
    __device__ __forceinline__ void read_t(float (&t)[T_ITEMS][8], int begin, int u0, int n) const
    {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int q = 0; q < T_ITEMS; ++q) {
            int line, unit;
            item_of_t(begin + q * T::NT < n * T::BM ? begin + q * T::NT : 0, n, line, unit);
            const int row = tile_row + line, k = (u0 + unit) * 8;
            const float *const p = a.T + (int64_t)(row < a.rows.M ? row : a.rows.M - 1) * a.ldt;
            if ((a.r & 7) == 0) {
                const f4 x = *(const f4 *)(p + k), y = *(const f4 *)(p + k + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { t[q][j] = x[j]; t[q][4 + j] = y[j]; }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[q][j] = p[k + j < a.r ? k + j : a.r - 1];
            }
        }
    }
    __device__ __forceinline__ void write_t(char *lds, float (&t)[T_ITEMS][8], int begin, int u0, int n) const
    {
#pragma unroll
        for (int q = 0; q < T_ITEMS; ++q) {
            if (begin + q * T::NT >= n * T::BM) return;
            int line, unit;
            item_of_t(begin + q * T::NT, n, line, unit);
            const int row = tile_row + line, k = (u0 + unit) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) t[q][j] = row < a.rows.M && k + j < a.r ? t[q][j] : 0.0f;
            for (int piece = 0; piece < kPieces; ++piece) {
                xt_u4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = bf16_pair(piece_of(t[q][2 * j], piece, kPieces), piece_of(t[q][2 * j + 1], piece, kPieces));
                *(xt_u4 *)(lds + ((unit * kPieces + piece) * T::BM + (line ^ turn(unit))) * 16) = v;
            }
        }
    }
    // from item `begin` of the thread's on
    __device__ __forceinline__ void lay_out_t(char *lds, int begin, int u0, int n) const
    {
        for (int at = (int)threadIdx.x + begin * T::NT; at < n * T::BM; at += T_ITEMS * T::NT) {
            float t[T_ITEMS][8];
            read_t(t, at, u0, n);
            write_t(lds, t, at, u0, n);
        }
    }
    // An instruction's products added to block m, in the rows lo .. hi - 1.  (Blocks that a segment has whole could do without the choice; a
    // branch for them gained nothing, and there is to be none between a matrix instruction and what reads its result.)
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
};

// The segments that rows first .. last - 1 meet, 64 at a time: their rows and adapters in the lanes
struct Meeting {
    int chunk, lo, hi, adapter;
    uint64_t which;
    bool more;
    __device__ __forceinline__ void start(const Segments &g, int first, int last, int lane)
    {
        chunk = g.S <= 64 ? 0 : segment_of(g, first, lane);
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

// From memory, row by row on the vector ALU: T's row times its adapter's B, in fp32.  Four lanes have 32 ranks of a column between them, so
// that neighbouring lanes read neighbouring bytes; a matrix operand's lanes have columns of their own, a cache line for every 16 bytes (and across,
// two columns to a lane: 208 x 4096 x 4096, a row to a segment, rank 32 29 us, a column to a lane and value 42);
// and the sums go to a tile of LDS beside the ring, from where they join the others in the end.  The k groups take the rows
// in turn; a batch of rows is on its way while the one before is multiplied, the first one is asked for before the first stages of X and W.
// (A decoding batch has an adapter to a row, and a matrix instruction for each would have one row of 16: 192 rows by rank 32 beside 4096 x
// 4096 took 33 us so.)
template <class T>
struct AddFromRows : Adapters<T> {
    static constexpr int ROWS = T::MI * 16, LDS = T::LDS + T::BM * T::BN * 4;
    static constexpr int AT = 2;   // rows of a batch
    static_assert(ROWS <= 64 && T::NI <= 2, "a lane to a row; two columns to a lane");
    enum { WHOLE, CUT, ACROSS };   // B along its rows, in whole units of 8 ranks or not; across
    struct Batch {
        xt_u4 b[AT][T::NI];
        float t[AT][8];
        int row[AT];   // of the wave's; -1: an empty place
    };
    mutable Batch batch;
    mutable uint64_t left;   // rows not yet taken
    uint64_t mine;           // this group's
    int adapter, kind;       // of row row0 + lane; -1: none
    uint32_t off[T::NI];
    const char *first;       // B at the wave's first column (across: at its own)
    bool last;               // across: the lane's first column is B's last one, the second of what it reads
    // Along, a lane has 8 ranks of columns lane / 4 + 16 ni, four lanes a column's 32; across, of NI neighbouring columns, lanes 16 apart theirs
    template <int KIND>
    __device__ __forceinline__ int ranks() const { return 8 * (KIND == ACROSS ? this->lane >> 4 : this->lane & 3); }

    __device__ __forceinline__ AddFromRows(const Adapters<T> &x) : Adapters<T>(x)
    {
        const UpArgs &a = this->a;
        const int lane = this->lane, row0 = this->row0;
        adapter = -1;
        mine = 0;
        if (a.r == 0 || a.rows.S == 0 || this->idle) return;
        const int row1 = row0 + ROWS < a.rows.M ? row0 + ROWS : a.rows.M, row = row0 + lane;
        Meeting m;
        m.start(a.rows, row0, row1, lane);
        for (;;) {
            for (uint64_t some = m.which; some; some &= some - 1) {
                const int at = __builtin_ctzll(some);
                const int lo = __builtin_amdgcn_readlane(m.lo, at), hi = __builtin_amdgcn_readlane(m.hi, at), g = __builtin_amdgcn_readlane(m.adapter, at);
                adapter = row >= lo && row < hi && row < row1 ? g : adapter;
            }
            if (!m.more) break;
            m.next(a.rows, row0, row1, lane);
        }
        const uint64_t all = __ballot(adapter >= 0);
        mine = T::WK == 1 ? all : __ballot(adapter >= 0 && __popcll(all & ((1ull << lane) - 1)) % T::WK == this->kg);
        kind = a.across ? ACROSS : (a.r & 7) == 0 ? WHOLE : CUT;
        const uint32_t ld = (uint32_t)a.ldb * 2u;
        const int c0 = this->col0 < a.mm.N ? this->col0 : a.mm.N - 1;
        first = (const char *)a.B + (a.across ? 0 : (int64_t)c0 * a.ldb) * 2;
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) {
            int c = this->col0 + ni * 16 + (lane >> 2);
            c = (c < a.mm.N ? c : a.mm.N - 1) - c0;
            off[ni] = (uint32_t)c * ld;
        }
        last = false;
        if (a.across) {   // (B has NI columns at least)
            const int c = this->col0 + (lane & 15) * T::NI, end = a.mm.N - T::NI;
            last = c > end;
            off[0] = (uint32_t)(last ? end : c) * 2u;
        }
        left = mine;
        if (kind == WHOLE) fetch<WHOLE>(batch, 0);
    }

    // The next rows' operands, ranks k .. k + 31.  (As many reads whatever there is, and no branch around one: the wait for a batch then need
    // not be one for the next.  An empty place reads the first row's and adapter's.)
    template <int KIND>
    __device__ __forceinline__ void fetch(Batch &x, int k) const
    {
        typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        const UpArgs &a = this->a;
        const int at = k + ranks<KIND>();   // the lane's first rank
        const bool in = at < a.r;
        const uint32_t ld = (uint32_t)a.ldb * 2u;
#pragma unroll
        for (int q = 0; q < AT; ++q) {
            const bool there = left != 0;
            const int row = there ? __builtin_ctzll(left) : 0;
            left &= left - 1;
            x.row[q] = there ? row : -1;
            const int g = there ? __builtin_amdgcn_readlane(adapter, row) : 0;
            const char *const base = first + (int64_t)g * a.group_b * 2;
            const float *const t = a.T + (int64_t)(this->row0 + row) * a.ldt;
            if constexpr (KIND == WHOLE) {
                const f4 y = *(const f4 *)(t + (in ? at : 0)), z = *(const f4 *)(t + (in ? at : 0) + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { x.t[q][j] = y[j]; x.t[q][4 + j] = z[j]; }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x.t[q][j] = t[at + j < a.r ? at + j : a.r - 1];
            }
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                if constexpr (KIND == WHOLE) x.b[q][ni] = __builtin_bit_cast(xt_u4, *(const u4 *)(base + off[ni] + (in ? at * 2 : 0)));
                else if constexpr (KIND == CUT) {
                    x.b[q][ni] = xt_u4{0, 0, 0, 0};
                    if (in) x.b[q][ni] = load_unit<2>(base + off[ni], at * 2, a.r * 2);
                }
            }
            if constexpr (KIND == ACROSS) {   // (two columns of a rank, or two ranks of a column, to a word)
                typedef uint32_t u1 __attribute__((aligned(2)));
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const char *const p = base + (int64_t)(at + j < a.r ? at + j : a.r - 1) * ld + off[0];
                    if constexpr (T::NI > 1) v[j] = *(const u1 *)p;
                    else v[j] = *(const uint16_t *)p;
                }
                if constexpr (T::NI > 1) {
                    x.b[q][0] = xt_u4{v[0], v[1], v[2], v[3]};
                    x.b[q][T::NI - 1] = xt_u4{v[4], v[5], v[6], v[7]};
                } else x.b[q][0] = xt_u4{v[0] | (v[1] << 16), v[2] | (v[3] << 16), v[4] | (v[5] << 16), v[6] | (v[7] << 16)};
            }
        }
    }
    __device__ __forceinline__ float *place(int row, int c) const
    {
        return (float *)(xt_smem + T::LDS) + (this->row0 - this->tile_row + row) * T::BN + this->col0 - this->tile_col + c;
    }
    template <int KIND>
    __device__ __forceinline__ void multiply(const Batch &x, int k) const
    {
        const UpArgs &a = this->a;
        const int lane = this->lane, n = a.r - k - ranks<KIND>();   // the lane's ranks
#pragma unroll
        for (int q = 0; q < AT; ++q) {
            if (x.row[q] < 0) continue;
            if constexpr (KIND == ACROSS) {
                float sum[T::NI] = {};
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int c = 0; c < T::NI; ++c) {
                        const uint32_t w = T::NI > 1 ? x.b[q][j / 4 % T::NI][j % 4] : x.b[q][0][j / 2];
                        const float b = T::NI > 1 ? half_of<T::ELEM>(c == 0 && last ? w >> 16 : w, c) : half_of<T::ELEM>(w, j % 2);
                        sum[c] = j < n ? __builtin_fmaf(x.t[q][j], b, sum[c]) : sum[c];
                    }
#pragma unroll
                for (int c = 0; c < T::NI; ++c) {
                    sum[c] += __shfl_xor(sum[c], 16);
                    sum[c] += __shfl_xor(sum[c], 32);
                    if (lane < 16) {
                        float *const to = place(x.row[q], lane * T::NI + c);
                        *to = k == 0 ? sum[c] : *to + sum[c];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                continue;
            }
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float b = half_of<T::ELEM>(x.b[q][ni][j / 2], j % 2);
                    if constexpr (KIND == WHOLE) sum = __builtin_fmaf(x.t[q][j], b, sum);
                    else sum = j < n ? __builtin_fmaf(x.t[q][j], b, sum) : sum;
                }
                if constexpr (KIND == WHOLE) sum = n > 0 ? sum : 0.0f;
                sum += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, sum), 0xb1, 0xf, 0xf, true));   // lanes 1 0 3 2
                sum += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, sum), 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
                if ((lane & 3) == 0) {
                    float *const to = place(x.row[q], ni * 16 + (lane >> 2));
                    *to = k == 0 ? sum : *to + sum;
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // (one row's values after the other's)
        }
    }
    template <int KIND>
    __device__ __forceinline__ void rows() const
    {
        for (int k = 0; k < this->a.r; k += 32) {
            if (k > 0 || KIND != WHOLE) {
                left = mine;
                fetch<KIND>(batch, k);
            }
            for (;;) {
                Batch next;
                if (left == 0) { multiply<KIND>(batch, k); break; }
                fetch<KIND>(next, k);
                multiply<KIND>(batch, k);
                if (left == 0) { multiply<KIND>(next, k); break; }
                fetch<KIND>(batch, k);
                multiply<KIND>(next, k);
            }
        }
    }
    // beside the first stages
    __device__ __forceinline__ void operator()(xt_f4 (&)[T::MI][T::NI]) const
    {
        if (mine == 0) return;
        if (kind == WHOLE) rows<WHOLE>();
        else if (kind == CUT) rows<CUT>();
        else rows<ACROSS>();
    }
    // ... and the sums that they are (the k groups have met since)
    __device__ __forceinline__ void finish(xt_f4 (&acc)[T::MI][T::NI]) const
    {
        if (this->a.r == 0 || this->a.rows.S == 0 || this->idle) return;
        const int lane = this->lane;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            const int row = mi * 16 + (lane & 15);
            const bool has = __shfl(adapter, row) >= 0;
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                const xt_f4 x = *(const xt_f4 *)place(row, col_of<T>(ni, lane));
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[mi][ni][v] += has ? x[v] : 0.0f;
            }
        }
    }
};

// Through LDS: T's pieces and B's (slot (unit * pieces + piece) of a segment has 16 bytes of every column).  While one batch of segments is
// multiplied the next one's B is on its way into registers.
template <class T>
struct AddFromLds : Adapters<T> {
    // behind the ring: the first segments that the tile meets, which its first wave looks up while the first stages are on their way
    struct List {
        int4 of[64];   // adapter, first row, last row + 1
        int n, chunk, more;
    };
    static constexpr int LDS = T::LDS + (int)sizeof(List), ROOM = T::LDS;
    static constexpr int OF_B = Adapters<T>::OF_B;
    static constexpr int ITEMS = 4;   // 16 bytes of B that a thread has on their way
    static_assert(ROOM >= 4 * (kPieces * T::BM + OF_B * T::BN) * 16 && ITEMS * T::NT >= 4 * T::BN, "four units of both");
    // T and the first segments' B are asked for before the sums begin, where there are registers for them
    static constexpr bool AHEAD = T::BM < 256;
    static constexpr int T_ITEMS = Adapters<T>::T_ITEMS;
    // units at a time, in fours as an instruction has them (fp16, 8192 x 8192 x 4096, rank 64 on 256 x 256 tiles, four and four of 8 / six and two: 567 / 604 us)
    static constexpr int FIT = ROOM / (kPieces * T::BM * 16 + OF_B * T::BN * 16), ASKED = ITEMS * T::NT / T::BN, MOST = (FIT < ASKED ? FIT : ASKED) & ~3;
    mutable xt_u4 next[ITEMS];
    mutable float t0[T_ITEMS][8];
    int units;
    __device__ __forceinline__ AddFromLds(const Adapters<T> &x) : Adapters<T>(x)
    {
        units = (this->a.r + 7) / 8;
        if (AHEAD && this->a.r > 0 && this->a.rows.S > 0) this->read_t(t0, (int)threadIdx.x, 0, units < MOST ? units : MOST);
    }
    // segments of a batch, one at least
    __device__ __forceinline__ int at_once(int n_units) const
    {
        const int room = (ROOM - n_units * kPieces * T::BM * 16) / (n_units * OF_B * T::BN * 16), items = ITEMS * T::NT / (n_units * T::BN);
        return room < items ? room : items;
    }
    static __device__ __forceinline__ List *list() { return (List *)(xt_smem + T::LDS); }

    __device__ __forceinline__ void write(const Meeting &m) const
    {
        if ((m.which >> this->lane) & 1) list()->of[__popcll(m.which & ((1ull << this->lane) - 1))] = int4{m.adapter, m.lo, m.hi, 0};
        if (this->lane == 0) {
            list()->n = __popcll(m.which);
            list()->chunk = m.chunk;
            list()->more = m.more;
        }
    }
    __device__ __forceinline__ int last_row() const { return this->tile_row + T::BM < this->a.rows.M ? this->tile_row + T::BM : this->a.rows.M; }
    // the sums' beginning: nothing is added yet
    struct Look {
        const AddFromLds &x;
        __device__ __forceinline__ void operator()(xt_f4 (&)[T::MI][T::NI]) const
        {
            const UpArgs &a = x.a;
            if ((!AHEAD && threadIdx.x >= 64) || a.r == 0 || a.rows.S == 0) return;
            Meeting m;
            m.start(a.rows, x.tile_row, x.last_row(), x.lane);
            if (threadIdx.x < 64) x.write(m);
            if constexpr (AHEAD) {
                // (lane j: the j-th segment's adapter)
                // (all lanes take part: those of no segment send to the last one, which a full list alone reads)
                const int to = (m.which >> x.lane) & 1 ? __popcll(m.which & ((1ull << x.lane) - 1)) : 63;
                const int adapter = __builtin_amdgcn_ds_permute(to * 4, m.adapter);
                const int met = __popcll(m.which), n_units = x.units < MOST ? x.units : MOST, once = x.at_once(n_units);
                x.read_batch(x.next, met < once ? met : once, 0, n_units, [&](int k) { return __shfl(adapter, k); });
            }
        }
    };
    // the first wave's: the list of the next 64 segments, or the first again
    __device__ __forceinline__ void look(int chunk) const
    {
        Meeting m;
        m.chunk = chunk;
        m.look(this->a.rows, this->tile_row, last_row(), this->lane);
        write(m);
    }

    __device__ __forceinline__ void operator()(xt_f4 (&acc)[T::MI][T::NI]) const
    {
        const UpArgs &a = this->a;
        if (a.r == 0 || a.rows.S == 0) return;
        const int t_unit = kPieces * T::BM * 16, b_unit = OF_B * T::BN * 16;
        __syncthreads();   // (the ring is read no more, and the list is there)
        const int first = __builtin_amdgcn_readfirstlane(list()->chunk);
        if (!__builtin_amdgcn_readfirstlane(list()->n | list()->more)) return;
        for (int u0 = 0; u0 < units; u0 += MOST) {
            const int n_units = units - u0 < MOST ? units - u0 : MOST, once = at_once(n_units);
            char *const lds_b = xt_smem + n_units * t_unit;
            const Ways ways(n_units, kPieces * OF_B);
            if (u0 > 0) {
                __syncthreads();
                if (threadIdx.x < 64 && __builtin_amdgcn_readfirstlane(list()->chunk) != first) look(first);
                __syncthreads();
            }
            for (bool begun = false;; begun = true) {
                const int met = __builtin_amdgcn_readfirstlane(list()->n), chunk = __builtin_amdgcn_readfirstlane(list()->chunk), more = __builtin_amdgcn_readfirstlane(list()->more);
                const auto adapter = [&](int s0) { return [s0](int k) { return list()->of[s0 + k].x; }; };
                if (met > 0 && (!AHEAD || begun || u0 > 0)) read_batch(next, met < once ? met : once, u0, n_units, adapter(0));
                if (!begun) {
                    if (AHEAD && u0 == 0) this->write_t(xt_smem, t0, (int)threadIdx.x, 0, n_units);
                    this->lay_out_t(xt_smem, AHEAD && u0 == 0 ? T_ITEMS : 0, u0, n_units);
                }
                for (int s0 = 0; s0 < met; s0 += once) {
                    const int n = met - s0 < once ? met - s0 : once, left = met - s0 - n;
                    write_batch(next, lds_b, n, n_units);
                    __syncthreads();
                    if (left > 0) read_batch(next, left < once ? left : once, u0, n_units, adapter(s0 + n));
                    if (!this->idle)
                        for (int k = 0; k < n; ++k) {
                            const int4 seg = list()->of[s0 + k];
                            const int lo = __builtin_amdgcn_readfirstlane(seg.y), hi = __builtin_amdgcn_readfirstlane(seg.z);
                            if (lo < this->row0 + T::MI * 16 && hi > this->row0) products(acc, lds_b + k * n_units * b_unit, lo, hi, ways);
                        }
                    __syncthreads();
                }
                if (!more) break;
                __syncthreads();       // (the list is read no more)
                if (threadIdx.x < 64) look(chunk + 64);
                __syncthreads();
            }
        }
    }
    // which item of a batch a thread's q-th one is: segment k of it, unit, column of the tile (neighbouring threads: neighbouring addresses)
    __device__ __forceinline__ bool item(int q, int n, int units, int &k, int &unit, int &line) const
    {
        const int at = (int)threadIdx.x + q * T::NT;
        if (this->a.across) {
            line = at % T::BN;
            const int x = at / T::BN;
            k = x / units;
            unit = x - k * units;
        } else {
            const int x = at / units;
            unit = at - x * units;
            line = x % T::BN;
            k = x / T::BN;
        }
        return at < n * units * T::BN;
    }
    // B of n segments' adapters (adapter(k): the k-th one's), units u0 .. u0 + units - 1, the tile's columns
    template <class Adapter>
    __device__ __forceinline__ void read_batch(xt_u4 (&v)[ITEMS], int n, int u0, int units, Adapter adapter) const
    {
        const UpArgs &a = this->a;
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            int k, unit, line;
            const bool there = item(q, n, units, k, unit, line);
            const int g = adapter(there ? k : 0);
            if (!there) continue;
            const int c = this->tile_col + line;
            v[q] = this->read_b((const char *)a.B + (int64_t)g * a.group_b * 2, c < a.mm.N ? c : a.mm.N - 1, u0 + unit);
        }
    }
    __device__ __forceinline__ void write_batch(const xt_u4 (&v)[ITEMS], char *lds, int n, int units) const
    {
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            int k, unit, line;
            if (!item(q, n, units, k, unit, line)) continue;
#pragma unroll
            for (int p = 0; p < OF_B; ++p) *(xt_u4 *)(lds + (((k * units + unit) * OF_B + p) * T::BN + (this->line_of_b(line) ^ this->turn(unit))) * 16) = this->piece_of_b(v[q], p);
        }
    }
    __device__ __forceinline__ void products(xt_f4 (&acc)[T::MI][T::NI], const char *lds_b, int lo, int hi, const Ways &ways) const
    {
        const int lane = this->lane, b = lane >> 4;
        const char *const t_row = xt_smem + (this->row0 - this->tile_row) * 16, *const b_row = lds_b + (this->col0 - this->tile_col) * 16;
        const int each = ways.each(), steps = ways.reads() * each;
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
            int unit, way;
            const int read = s / each;
            const bool there = ways.at(read, s - read * each, b, unit, way);
            const int at = ((lane & 15) ^ this->turn(unit)) * 16;
            const char *const t_at = t_row + (there ? unit * kPieces + way / OF_B : 0) * (T::BM * 16) + at;
            const char *const b_at = b_row + (there ? unit * OF_B + way % OF_B : 0) * (T::BN * 16) + at;
            xt_u4 vb[T::NI];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                vb[ni] = *(const xt_u4 *)(b_at + ni * 256);
                if (!there) vb[ni] = xt_u4{0, 0, 0, 0};
            }
            for_each<T::MI>([&](auto mi) { this->template add_block<decltype(mi)::value>(acc, t_at, there, lo, hi, vb); });
        }
    }
};

template <class T, bool ROWS>
using AddAdapters = std::conditional_t<ROWS, AddFromRows<T>, AddFromLds<T>>;

template <class T, bool ROWS>
__global__ void __launch_bounds__(T::NT) __attribute__((amdgpu_waves_per_eu(!ROWS && T::BM * T::BN <= 64 * 64 ? 3 : 2))) adapters_up_kernel(const UpArgs u)
{
    static_assert(!T::AKS && !T::FP8 && (ROWS || T::WK == 1), "16-bit products by rows");
    static_assert(AddAdapters<T, ROWS>::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
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
    const AddAdapters<T, ROWS> adapters(Adapters<T>{u, row0, col0, wave_row, wave_col, lane, kg, idle});
    if constexpr (ROWS) {
        if (!tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc, adapters)) return;
        adapters.finish(acc);
    } else {
        tile_sums<T>(sa, sb, 0, a.K, wave, kg, lane, a_row, TileScales(), idle, acc, typename AddFromLds<T>::Look{adapters});
        adapters(acc);
    }
    store_sums<T>(acc, a.R, a.out, lane, wave_col, from, a.N, [&](int mi) -> int64_t {
        const int i = wave_row + mi * 16 + (lane & 15);
        return i < a.M ? (int64_t)i * a.ldr : -1;
    });
}

template <class T, bool ROWS>
inline hipError_t launch_adapters_tile(const UpArgs &a, int64_t blocks, hipStream_t s)
{
    constexpr int lds = AddAdapters<T, ROWS>::LDS;
    if (blocks <= 0) return hipSuccess;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    static const hipError_t granted = hipFuncSetAttribute((const void *)adapters_up_kernel<T, ROWS>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
    adapters_up_kernel<T, ROWS><<<dim3((unsigned)blocks), dim3(T::NT), lds, s>>>(a);
    return hipGetLastError();
}

template <int ELEM, bool BKS>
inline hipError_t launch_adapters_layout(int tile, bool many, const UpArgs &a, int64_t blocks, hipStream_t s)
{
    switch (tile) {
    case EXPERTS_256x256: return launch_adapters_tile<ExpertTile<ELEM, 256, 256, 2, 4, 1, 2, false, BKS>, false>(a, blocks, s);
    case EXPERTS_128x128: return launch_adapters_tile<ExpertTile<ELEM, 128, 128, 2, 2, 1, 2, false, BKS>, false>(a, blocks, s);
    case EXPERTS_64x128: return launch_adapters_tile<ExpertTile<ELEM, 64, 128, 2, 2, 1, 3, false, BKS>, false>(a, blocks, s);
    case EXPERTS_64x64: {
        typedef ExpertTile<ELEM, 64, 64, 2, 2, 1, 3, false, BKS> T;
        return many ? launch_adapters_tile<T, true>(a, blocks, s) : launch_adapters_tile<T, false>(a, blocks, s);
    }
    case EXPERTS_64x64_K2: return launch_adapters_tile<ExpertTile<ELEM, 64, 64, 2, 2, 2, 3, false, BKS>, true>(a, blocks, s);
    case EXPERTS_16x32: return launch_adapters_tile<ExpertTile<ELEM, 16, 32, 1, 1, 4, 3, false, BKS>, true>(a, blocks, s);
    default: return launch_adapters_tile<ExpertTile<ELEM, 16, 16, 1, 1, 8, 4, false, BKS>, true>(a, blocks, s);
    }
}

// many: segments of a few rows; the tile is EXPERTS_64x64 or smaller then
template <int ELEM>
inline hipError_t launch_adapters_up(int tile, bool w_across, bool many, const UpArgs &a, int64_t blocks, hipStream_t s)
{
    return w_across ? launch_adapters_layout<ELEM, true>(tile, many, a, blocks, s) : launch_adapters_layout<ELEM, false>(tile, many, a, blocks, s);
}

}  // namespace amulet
#endif
