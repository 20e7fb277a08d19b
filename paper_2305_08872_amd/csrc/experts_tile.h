// Matrix products by groups of rows, 16-bit and 8-bit floating point operands, on the matrix cores:
//     R[i][:] = A[row(i)][:] B[g(i)]                        by rows  (experts' products and their rows' gradients)
//     R[g]    = sum over the rows i of g of A[row(i)]^T D[i]  by sums (the gradients of the experts' weights)
// One kernel body for both; the translation units experts_mm_*.hip hold its instances.
//
// A stage of an operand is 128 bytes of k per line (64 k of 16 bits, 128 of 8), streamed global -> LDS by
// global_load_lds_dwordx4 (64 lanes x 16 bytes, any byte alignment) through a ring of S stages.  Two storages:
//   k along the rows (KC): LDS keeps [line][units of 16 bytes]; a lane's fragment is one ds_read_b128.
//   k across them   (KS): LDS keeps [k][line], and ds_read_b64_tr_b16 / _b8 hand a lane the k of its line.
// Both are XOR-swizzled by unit so that the lanes of an LDS clock fall on distinct banks (unit_of below).  A stage that
// does not lie wholly inside its operand (the last k, lines past the edge that end inside a unit) goes through registers
// instead, element by element, with zeros past the end: nothing outside an operand is read.  (Of a whole stage a unit that the edge
// cuts is read whole; what it reads past its row lies in rows behind it, see stages_of_whole_units.)
//
// The matrix instruction takes B's lines as its rows and A's as its columns, so that a lane ends up with neighbouring
// columns of one row of R.  Sums are fp32; fp8 operands have one scale per 128 k, so an instruction's 16 x 16 x 128 products
// are summed alone and then added to the accumulators times both scales.
//
// What bounds them.  Few rows: the matrices' bytes (48 rows over 64 groups of 2048 x 2048, all busy ones read once: 58 us, 4.8 TB/s of
// a large copy's 4.95).  Many rows: the matrix cores, which the 256 x 256 tile keeps busy 60 to 70 % of its time (bf16 32768 x 4096 x
// 4096 over 32 ragged groups 1040 us = 1057 TFLOP/s, 8 bits over 16 643 us = 1710; a large library product of one matrix 1350 and 2602).
// The rest is power (the instructions alone reach 2050 TFLOP/s on normal bf16 values, 2450 on zeros; with the operands' way beside them
// the clock is 1.7 GHz), the tile's start and end (8 us where nothing else runs on the unit: LDS holds one such tile), and ragged
// groups' last tiles.  In between, few tiles: a stage's way from memory (a microsecond), of which a unit has 128 to 144 KB under way.
//
// Why these tiles: of the LDS, 2 x 64 KB of stages for 256 x 256 (an operand byte is read from L2 once per 256 lines), the smaller ones two or
// three workgroups to a unit so that one's start lies under another's products; 16 x 32 with four k groups for a
// handful of rows, where more workgroups draw more of the memory (57 us for the 48 rows above; 128 x 128 63).
// LDS bank conflicts: none counted in any of them, by rows or by sums, bf16 and 8 bits, B in either storage.
#ifndef AMULET_EXPERTS_TILE_H
#define AMULET_EXPERTS_TILE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "experts_internal.h"

// the LDS-DMA asm below sets M0 itself and says so in its clobber list
#pragma clang diagnostic ignored "-Winline-asm"

namespace amulet {

typedef float xt_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t xt_u4 __attribute__((ext_vector_type(4)));
typedef uint32_t xt_u2 __attribute__((ext_vector_type(2)));
typedef int xt_i8 __attribute__((ext_vector_type(8)));
typedef short xt_s4 __attribute__((ext_vector_type(4)));
typedef int xt_i2 __attribute__((ext_vector_type(2)));
typedef __bf16 xt_bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 xt_h8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) xt_s4 *xt_lds_s4;
typedef __attribute__((address_space(3))) xt_i2 *xt_lds_i2;
typedef __attribute__((address_space(3))) void *xt_lds_void;

extern __shared__ __attribute__((aligned(16))) char xt_smem[];

template <int ELEM_, int BM_, int BN_, int WM_, int WN_, int WK_, int S_, bool AKS_, bool BKS_>
struct ExpertTile {
    static constexpr int ELEM = ELEM_;                       // EXPERTS_BF16, _FP16, _FP8, _FP8_EXACT
    static constexpr bool FP8 = ELEM == EXPERTS_FP8 || ELEM == EXPERTS_FP8_EXACT;
    static constexpr int ES = FP8 ? 1 : 2;                   // bytes of an element
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WK = WK_, S = S_;
    static constexpr bool AKS = AKS_, BKS = BKS_;
    static constexpr int KB = 128, BK = KB / ES;             // bytes and k of a stage's line
    static constexpr int NW = WM * WN, NT = 64 * NW * WK;    // waves of a k group; threads
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int A_BYTES = BM * KB, B_BYTES = BN * KB;
    static constexpr int SA_BYTES = FP8 ? (BM < 64 ? 256 : BM * 4) : 0;   // scales of A's rows
    static constexpr int STAGE = A_BYTES + B_BYTES + SA_BYTES;
    static constexpr bool TURN = BM >= 256 && !AKS && !FP8;   // where the k begin, see tile_sums
    static constexpr int SPREAD = BM >= 256 && !FP8 ? 2 : 0;   // matrix instructions between those of a request
    static constexpr int PREFETCH = BM >= 256 && AKS ? 2 : 0;      // stages further on whose lines are asked for ahead, see tile_sums
    static constexpr int LDS = S * STAGE * WK + (PREFETCH ? 256 : 0);
    // neighbouring fragments of B interleave their columns, so that a lane's values of both are 8 in a row
    static constexpr bool PERM = !BKS && NI % 2 == 0;
    // the largest tile has registers for 32-bit offsets of A's rows only (its caller sees to it that they fit)
    static constexpr bool WIDE = BM < 256;
    static constexpr bool ALWAYS = BM >= 256;   // requests past the end, see tile_sums
    // the last k as a whole stage moved back, see tile_sums.  (Not the largest tile by rows: 8 bits leave no registers for the masks, and with 16 the
    // other stages took 0.8 % longer; by sums, where every group has such an end, 666 / 653 us for the two gradients of 16384 x 4096 x 2048.)
    static constexpr bool BACK = BM < 256 || AKS;
    static_assert(WK == 1 || BM < 256, "the largest tile has no room for k groups");
};

// Position of 16-byte unit `u` of LDS line `line` (RB bytes long); see the two storages above.  256 bytes hold 16 units,
// the banks of one clock:
//   KC, natural fragments (lines 0..15 at one u): 2 lines per 256 bytes, so bits 1..3 of the line;
//   KC, interleaved (lines 8 a + c, a, c = 0..3, or + 4): bits 1 and 3, 4;
//   KS: 16-bit reads take 32 bytes of rows {0..3, 8..11} at a time, 8-bit reads 16 of rows {0..7, 16..23}.
template <int RB, bool KS, bool PERM, int ES>
__device__ __forceinline__ int unit_of(int line, int u)
{
    if constexpr (!KS) return u ^ (PERM ? ((line >> 2) & 6) | ((line >> 1) & 1) : (line >> 1) & 7);
    else if constexpr (ES == 2) {
        if constexpr (RB >= 256) return u ^ (((line & 3) | ((line >> 1) & 4)) << 1);
        else if constexpr (RB == 128) return u ^ ((((line >> 1) & 1) | ((line >> 2) & 2)) << 1);
        else if constexpr (RB == 64) return u ^ (((line >> 3) & 1) << 1);
        else return u;
    } else {
        if constexpr (RB >= 256) return u ^ ((line & 7) | ((line >> 1) & 8));
        else if constexpr (RB == 128) return u ^ (((line >> 1) & 3) | ((line >> 2) & 4));
        else if constexpr (RB == 64) return u ^ (((line >> 2) & 1) | ((line >> 3) & 2));
        else if constexpr (RB == 32) return u ^ ((line >> 4) & 1);
        else return u;
    }
}

__device__ __forceinline__ void dma16(const char *p, uint32_t lds)
{
    lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory", "m0");
}
// a pointer that is the same in all lanes, in scalar registers
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t x = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)x), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32));
    return (const char *)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ void dma16(const char *base, uint32_t off, uint32_t lds)
{
    base = uniform(base);
    lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const char *base, uint32_t off, uint32_t lds)
{
    base = uniform(base);
    lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}

// what an index that names no row stands for
__device__ const xt_u4 xt_zeros = {0, 0, 0, 0};

// 16 bytes of a storage row of `end` bytes (at least one of them) from byte `at` on, zeros past its end.  Where they cross it the row's
// last 16 are read and moved down: one load, nothing outside the row.
template <int ES>
__device__ __forceinline__ xt_u4 load_unit(const char *row, int at, int end)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(1)));
    xt_u4 v = {0, 0, 0, 0};
    if (end >= 16) {
        const int from = at + 16 <= end ? at : end - 16, down = at - from;   // bytes
        const u4 x = *(const u4 *)(row + from);
        unsigned __int128 w = ((unsigned __int128)(((uint64_t)x[3] << 32) | x[2]) << 64) | (((uint64_t)x[1] << 32) | x[0]);
        w = down < 16 ? w >> (8 * down) : 0;
        v = xt_u4{(uint32_t)w, (uint32_t)(w >> 32), (uint32_t)(w >> 64), (uint32_t)(w >> 96)};
    } else {
#pragma unroll
        for (int i = 0; i < 16 / ES; ++i) {
            const int b = at + i * ES;
            const uint32_t x = b >= end ? 0u : ES == 2 ? (uint32_t) * (const uint16_t *)(row + b) : (uint32_t) * (const uint8_t *)(row + b);
            v[i * ES / 4] |= x << (8 * ((i * ES) % 4));
        }
    }
    return v;
}

// One operand on its way into LDS: LINES lines (rows of A, columns of B), one stage at a time, by the NW waves of a k group.
// The LDS units of a stage are loaded 64 by a wave instruction: instruction j of the stage, j = wave + NW q.  An address is a
// base in scalar registers that moves on by stages and 32 bits per lane that stay; WIDE: 64 bits per lane (rows given by an
// index may lie further apart).  A KS operand with an index has its storage rows read a stage ahead.
template <int LINES, int ES, int KB, bool KS, bool PERM, int NW, bool WIDE>
struct Staged {
    static constexpr int LOADS = LINES * KB / 1024;                           // instructions of a stage, all waves
    static constexpr int Q = (LOADS + NW - 1) / NW;                           // ... of one wave (the last waves may repeat others')
    static constexpr int RB = KS ? LINES * ES : KB, UR = RB / 16;             // bytes, units of an LDS line
    static constexpr int E = 16 / ES;

    const char *first;       // storage at the group's first k (KS) or at line 0 (KC)
    const char *base;        // ... at the next stage to load
    int64_t pitch;           // bytes between storage rows
    const int32_t *index;    // KS: storage row of a k, or null: the k itself
    const char *p[WIDE && !KS ? Q : 1];
    uint32_t off[WIDE && !KS ? 1 : Q];
    int row[KS ? Q : 1];     // KS with an index: the next stage's
    int lines, line0;        // lines of the operand, the tile's first
    int k, storage_rows;     // k of the group; rows that an index may name

    static __device__ __forceinline__ int slot(int q, int wave, int lane) { return ((wave + NW * q) % LOADS) * 64 + lane; }

    // `row_of(line)`: storage row of a line that is inside
    template <class RowOf>
    __device__ __forceinline__ void start_kc(const char *b, int64_t pitch_bytes, int first_line, int n, int k_all, int k0, int wave, int lane, RowOf row_of, bool relative)
    {
        first = b; pitch = pitch_bytes; lines = n; line0 = first_line; k = k_all; index = nullptr; storage_rows = 0;
        // (relative: lines are storage rows, and the offsets count from the tile's first)
        base = b + (relative && !WIDE ? (int64_t)first_line * pitch_bytes : 0) + (int64_t)k0 * ES;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int s = slot(q, wave, lane), line = s / UR, u = unit_of<RB, false, PERM, ES>(line, s % UR);
            const int in = first_line + line < n ? first_line + line : n - 1;
            if constexpr (WIDE) p[q] = base + (int64_t)row_of(in) * pitch_bytes + u * 16;
            else off[q] = (uint32_t)(row_of(in) - (relative ? first_line : 0)) * (uint32_t)pitch_bytes + (uint32_t)(u * 16);
        }
    }
    __device__ __forceinline__ void start_ks(const char *b, int64_t pitch_bytes, const int32_t *idx, int rows, int first_line, int n, int k_all, int k0, int wave, int lane)
    {
        first = b; pitch = pitch_bytes; lines = n; line0 = first_line; k = k_all; index = idx; storage_rows = rows;
        base = b + (idx ? 0 : (int64_t)k0 * pitch_bytes);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int s = slot(q, wave, lane), r = s / UR;
            off[q] = (uint32_t)column_of(r, s % UR) + (idx ? 0u : (uint32_t)r * (uint32_t)pitch_bytes);
        }
        if (idx) read_index(k0, wave, lane);
    }
    __device__ __forceinline__ void read_index(int k0, int wave, int lane)
    {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int at = k0 + slot(q, wave, lane) / UR;
            row[KS ? q : 0] = at < k ? index[at] : -1;
        }
    }
    // byte offset in a storage row of the unit at LDS place `place` of line `r` (past the edge: the last whole unit, whose values nobody stores)
    __device__ __forceinline__ int64_t column_of(int r, int place) const
    {
        int c = line0 + unit_of<RB, KS, PERM, ES>(r, place) * E;
        c = c < lines ? c : (lines - 1) / E * E;
        return (int64_t)c * ES;
    }
    // whether some unit of the tile holds lines on both sides of the edge: read whole it ends outside its row
    __device__ __forceinline__ bool cut() const { return KS && line0 + LINES > lines && lines % E != 0; }

    // instruction q of the whole stage that is next, into `lds`
    template <int q>
    __device__ __forceinline__ void load(uint32_t lds, int wave)
    {
        const uint32_t to = lds + (uint32_t)((wave + NW * q) % LOADS) * 1024u;
        if constexpr (KS) {
            if (index) {
                const int r = row[q];
                const char *const from = base + (int64_t)r * pitch + off[q];
                dma16((unsigned)r < (unsigned)storage_rows ? from : (const char *)&xt_zeros, to);
                return;
            }
        }
        if constexpr (WIDE && !KS) dma16(p[q], to);
        else dma16(base, off[q], to);
    }
    // on to the stage at k0
    __device__ __forceinline__ void advance(int k0, int ahead, int wave, int lane)
    {
        if (KS && index) { read_index(k0, wave, lane); return; }
        if constexpr (WIDE && !KS)
#pragma unroll
            for (int q = 0; q < Q; ++q) p[q] += ahead * ES;
        else base += KS ? (int64_t)ahead * pitch : (int64_t)ahead * ES;
    }
    // KS, lane `at` of LINES: offset of one of the 128-byte lines that a stage is read from
    __device__ __forceinline__ uint32_t line_of(int at) const
    {
        static_assert(KS, "lines of k across the storage");
        constexpr int PER = RB / 128;
        int c = line0 * ES + at % PER * 128;
        c = c < lines * ES ? c : 0;
        return (uint32_t)(at / PER) * (uint32_t)pitch + (uint32_t)c;
    }
    // the stage at k0, of which any part may be there, through registers
    template <class RowOf>
    __device__ __forceinline__ void load_cut(char *lds, int k0, int wave, int lane, RowOf row_of)
    {
        // (two units of a lane at a time: more would not fit beside the largest tile's accumulators)
        constexpr int AT = Q > 1 ? 2 : 1;
        static_assert(Q % AT == 0, "units in pairs");
#pragma unroll 1
        for (int q0 = 0; q0 < Q; q0 += AT) {
            xt_u4 v[AT];
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const int s = slot(q0 + i, wave, lane);
                v[i] = xt_u4{0, 0, 0, 0};
                if constexpr (!KS) {
                    const int line = s / UR, at = k0 + unit_of<RB, false, PERM, ES>(line, s % UR) * E;
                    const int in = line0 + line < lines ? line0 + line : lines - 1;
                    if (at < k) v[i] = load_unit<ES>(first + (int64_t)row_of(in) * pitch, at * ES, k * ES);
                } else {
                    const int r0 = s / UR, c = line0 + unit_of<RB, KS, PERM, ES>(r0, s % UR) * E;
                    if (k0 + r0 < k && c < lines) {
                        int r = k0 + r0;
                        bool there = true;
                        if (index) { r = index[r]; there = (unsigned)r < (unsigned)storage_rows; }
                        if (there) v[i] = load_unit<ES>(first + (int64_t)r * pitch, c * ES, lines * ES);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < AT; ++i) *(xt_u4 *)(lds + slot(q0 + i, wave, lane) * 16) = v[i];
        }
    }
};

// Fragments: a lane's 16 bytes of half `h` of a stage, of the fragment that starts at line f (KC) or at its columns (KS).
template <class T, int LINES, bool KS, bool PERM>
struct FragReader {
    static constexpr int ES = T::ES, RB = KS ? LINES * ES : T::KB;
    int at[2];       // KC: byte offset of this lane's unit, of each half (units b and b + 4: the swizzle does not change bit 2)
    int row, part;   // KS: this lane's first row; half unit (16 bits: 8 bytes of four)
    int wave0;       // the wave's first line
    // i: fragment line of the lane, b: k block of the lane
    __device__ __forceinline__ void start(int first_line, int lane)
    {
        const int i = lane & 15, b = lane >> 4;
        wave0 = first_line;
        if constexpr (!KS) {
            const int line = first_line + (PERM ? 8 * (i >> 2) + (i & 3) : i);
            at[0] = line * RB + unit_of<RB, false, PERM, ES>(line, b) * 16;
            at[1] = at[0] ^ 64;
        } else if constexpr (ES == 2) {
            row = 8 * b + (i >> 2);
            part = i & 3;
        } else {
            row = 16 * b + (i >> 1);
            part = i & 1;
        }
    }
    // half h (64 bytes of k) of fragment f
    __device__ __forceinline__ xt_u4 read(const char *lds, int f, int h) const
    {
        if constexpr (!KS) {
            // (nor does it change with the fragment: its lines are a constant further on)
            const int line = PERM ? (f >> 1) * 32 + (f & 1) * 4 : f * 16;
            return *(const xt_u4 *)(lds + at[h] + line * RB);
        } else if constexpr (ES == 2) {
            xt_u4 v;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int r = row + 4 * t + 32 * h;
                const int u = unit_of<RB, true, false, 2>(r, (wave0 + 16 * f) / 8 + (part >> 1));
                const xt_s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((xt_lds_s4)(lds + r * RB + u * 16 + (part & 1) * 8));
                const xt_u2 y = __builtin_bit_cast(xt_u2, x);
                v[2 * t] = y[0];
                v[2 * t + 1] = y[1];
            }
            return v;
        } else {
            xt_u4 v;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int r = row + 8 * t + 64 * h;
                const int u = unit_of<RB, true, false, 1>(r, (wave0 + 16 * f) / 16);
                const xt_i2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((xt_lds_i2)(lds + r * RB + u * 16 + part * 8));
                v[2 * t] = (uint32_t)x[0];
                v[2 * t + 1] = (uint32_t)x[1];
            }
            return v;
        }
    }
};

template <int ELEM>
__device__ __forceinline__ xt_f4 mma16(xt_u4 a, xt_u4 b, xt_f4 c)
{
    if constexpr (ELEM == EXPERTS_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(xt_bf8, a), __builtin_bit_cast(xt_bf8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(xt_h8, a), __builtin_bit_cast(xt_h8, b), c, 0, 0, 0);
}

// eight e4m3 values of a unit (its first or second half) as bf16, exactly
__device__ __forceinline__ xt_u4 bf16_of(xt_u4 x, int half)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    xt_u4 y;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = x[2 * half + i];
        const bf2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
        y[2 * i] = __builtin_bit_cast(uint32_t, lo);
        y[2 * i + 1] = __builtin_bit_cast(uint32_t, hi);
    }
    return y;
}

// V consecutive values of R from column c on, those of columns `from` to `cols` - 1; rounded once, to the output's type.
// (Vector stores whatever the address: 5 x 2341 x 457 over 33 groups, rows at odd multiples of two bytes.)
template <int V>
__device__ __forceinline__ void store_out(void *R, int out, int64_t row_at, int c, int from, int cols, const float *x)
{
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
    typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
    if (c >= cols || c + V <= from) return;
    const bool whole = c >= from && c + V <= cols;
    if (out == EXPERTS_FP32) {
        float *p = (float *)R + row_at + c;
        if (whole) {
#pragma unroll
            for (int i = 0; i < V; i += 4) *(f4 *)(p + i) = f4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i >= from && c + i < cols) p[i] = x[i];
        }
        return;
    }
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        uint16_t lo, hi;
        if (out == EXPERTS_BF16) {
            lo = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
            hi = __builtin_bit_cast(uint16_t, (__bf16)x[i + 1]);
        } else {
            lo = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
            hi = __builtin_bit_cast(uint16_t, (_Float16)x[i + 1]);
        }
        w[i / 2] = lo | ((uint32_t)hi << 16);
    }
    uint16_t *p = (uint16_t *)R + row_at + c;
    if (whole) {
        if constexpr (V == 8) *(u4 *)p = u4{w[0], w[1], w[2], w[3]};
        else *(u2 *)p = u2{w[0], w[1]};
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (c + i >= from && c + i < cols) p[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    }
}

// Which tile a workgroup has.  Row tiles of the groups in order, then those of the rows before the first group and behind
// the last one, which are zeros (group -1).  Every wave finds it for itself: lane l looks at group l.
struct RowTile {
    int group, row0, row1, tm, tn;
};
__device__ __forceinline__ int clamp_row(int x, int M) { return x < 0 ? 0 : x > M ? M : x; }
// Tile `in` of a region of `high_all` row tiles: panels of 8 row tiles, column by column.  (Unsigned 32-bit divisions: a grid
// has fewer than 2^23 workgroups.)
__device__ __forceinline__ void tile_in_region(uint32_t in, uint32_t high_all, uint32_t tiles_n, int &tm, int &tn)
{
    const uint32_t panel = in / (8 * tiles_n), rem = in - panel * 8 * tiles_n;
    const uint32_t high = high_all - panel * 8 < 8 ? high_all - panel * 8 : 8, col = rem / high;
    tm = (int)min(panel * 8 + rem - col * high, high_all - 1);   // (inside in any case: offsets that do not ascend may count more tiles than 32 bits)
    tn = (int)min(col, tiles_n - 1);
}
// A launch that has a part of the columns: `tiles_n` becomes its own, and how many tiles lie before them.  rows: of 256 x 256 tiles.
template <int BM>
__device__ __forceinline__ int own_columns(const ExpertsArgs &a, uint32_t rows, int &tiles_n)
{
    if (BM < 128 || !a.part_of) return 0;
    const int before = columns_of_largest(rows, (a.N + 255) / 256, a.units, a.gap) * (256 / BM);   // (square tiles only)
    if (a.part_of == EXPERTS_BEFORE) { tiles_n = tiles_n < before ? tiles_n : before; return 0; }
    tiles_n = tiles_n > before ? tiles_n - before : 0;
    return before;
}
template <int BM>
__device__ __forceinline__ bool find_row_tile(const ExpertsArgs &a, int tiles_n, uint32_t block, RowTile &t)
{
    // XCD x (workgroup b runs on XCD b % 8) takes an eighth of the tiles, neighbours in the order of regions
    const uint32_t xcd = block & 7, slot = block >> 3;
    if (!a.offsets) {
        const uint32_t high = (uint32_t)(a.M + BM - 1) / BM;
        const int skipped = own_columns<BM>(a, (uint32_t)(a.M + 255) / 256, tiles_n);
        const uint32_t tiles = high * (uint32_t)tiles_n;
        const uint32_t begin = (uint32_t)((uint64_t)tiles * xcd >> 3), end = (uint32_t)((uint64_t)tiles * (xcd + 1) >> 3);
        if (slot >= end - begin) return false;
        t.group = 0;
        t.row0 = 0;
        t.row1 = a.M;
        tile_in_region(begin + slot, high, (uint32_t)tiles_n, t.tm, t.tn);
        t.tn += skipped;
        return true;
    }
    const int lane = threadIdx.x & 63;
    const int regions = a.G + 2;
    auto region = [&](int g, int &lo, int &hi) {
        if (g < a.G) { lo = clamp_row(a.offsets[g], a.M); hi = clamp_row(a.offsets[g + 1], a.M); }
        else if (g == a.G) { lo = 0; hi = clamp_row(a.offsets[0], a.M); }
        else if (g == a.G + 1) { lo = clamp_row(a.offsets[a.G], a.M); hi = a.M; }
        else lo = hi = 0;
    };
    auto scan = [&](int c, int &lo, int &hi, int &n) {   // row tiles of regions c .. c + lane
        region(c + lane, lo, hi);
        n = hi > lo ? (hi - lo + BM - 1) / BM : 0;
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        return sum;
    };
    int lo, hi, n;
    int first = scan(0, lo, hi, n);
    uint32_t total = (uint32_t)__builtin_amdgcn_readlane(first, 63);
    for (int c = 64; c < regions; c += 64) {
        int l2, h2, n2;
        total += (uint32_t)__builtin_amdgcn_readlane(scan(c, l2, h2, n2), 63);
    }
    uint32_t largest = total;   // rows of 256 x 256 tiles
    if (BM == 128 && a.part_of) {
        int sum = 0;
        for (int c = 0; c < regions; c += 64) {
            int l2, h2;
            region(c + lane, l2, h2);
            sum += h2 > l2 ? (h2 - l2 + 255) / 256 : 0;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        largest = (uint32_t)__builtin_amdgcn_readfirstlane(sum);
    }
    const int skipped = own_columns<BM>(a, largest, tiles_n);
    const uint64_t tiles = (uint64_t)total * (uint32_t)tiles_n;
    const uint32_t begin = (uint32_t)(tiles * xcd >> 3), end = (uint32_t)(tiles * (xcd + 1) >> 3);
    if (slot >= end - begin) return false;
    const uint32_t at = begin + slot;
    // the region that holds tile `at`
    uint32_t before = 0;
    int c = 0;
    for (;;) {
        const uint64_t past = __ballot((uint64_t)(before + (uint32_t)first) * (uint32_t)tiles_n > at);
        if (past) {
            const int l = __builtin_ctzll(past);
            const uint32_t nl = (uint32_t)__builtin_amdgcn_readlane(n, l), upto = (uint32_t)__builtin_amdgcn_readlane(first, l);
            if (nl == 0) return false;
            t.group = c + l < a.G ? c + l : -1;
            t.row0 = __builtin_amdgcn_readlane(lo, l);
            t.row1 = __builtin_amdgcn_readlane(hi, l);
            tile_in_region(at - (before + upto - nl) * (uint32_t)tiles_n, nl, (uint32_t)tiles_n, t.tm, t.tn);
            t.tn += skipped;
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane(first, 63);
        c += 64;
        if (c >= regions) return false;   // (never: the tiles counted above are there)
        first = scan(c, lo, hi, n);
    }
}

// A wave's products of one stage, in steps: 16 bits: each instruction's k times halves of the wave's rows; 8 bits: one or two row
// blocks (an instruction has all 128 k).  While a step's matrix instructions run, the next one's fragments are read, into
// the other of two sets of registers.
template <class T>
struct Steps {
    static constexpr int KSTEPS = T::FP8 ? 1 : T::KB / 64;
    static constexpr int MA = T::FP8 ? (T::MI > 1 && T::MI < 8 ? 2 : 1) : T::MI > 1 ? T::MI / 2 : 1;   // row blocks of a step
    static constexpr int MSTEPS = T::MI / MA, STEPS = KSTEPS * MSTEPS;
    static constexpr bool A2 = STEPS % 2 == 0;   // (one step of 8 bits: read when the stage before is done with)
    static constexpr bool B2 = !T::FP8;          // (8 bits: one set, two would not leave room for the accumulators)
    static_assert(!B2 || KSTEPS == 2, "a stage begins with the first set");
    typedef FragReader<T, T::BM, T::AKS, false> ReadA;
    typedef FragReader<T, T::BN, T::BKS, T::PERM> ReadB;
    static constexpr int U = T::FP8 ? 2 : 1;     // 16-byte halves of a fragment

    // 8 bits, the largest tile: the rows' first half step by step, the second half column by column (stage_split)
    static constexpr bool SPLIT = T::FP8 && T::MI == 8;

    xt_u4 a[2][MA][U];
    xt_u4 b[B2 ? 2 : 1][T::NI][U];
    float w[2][MA];                              // fp8: the rows' scales
    xt_u4 rest[SPLIT ? T::MI / 2 : 1][U];        // (SPLIT: the second half's fragments and scales)
    float rest_w[SPLIT ? T::MI / 2 : 1];

    template <int j>
    __device__ __forceinline__ void read_rest(const ReadA &r, const char *la, const float *scales)
    {
        rest[j][0] = r.read(la, T::MI / 2 + j, 0);
        rest[j][U - 1] = r.read(la, T::MI / 2 + j, 1);
        rest_w[j] = scales[(T::MI / 2 + j) * 16];
    }
    __device__ __forceinline__ void read_b_one(const ReadB &r, const char *lb, int ni)
    {
        b[0][ni][0] = r.read(lb, ni, 0);
        b[0][ni][U - 1] = r.read(lb, ni, 1);
    }
    // one instruction of 128 k, added up times f.  (EXPERTS_FP8: its sum keeps some 17 bits below the largest product, not fp32's 24.  Taken
    // for results of 16 bits only: it costs 1.5e-5 of a sum where they round by 3e-4 or more; where a block's large products cancel
    // the loss shows, up to 2^-10 of the largest, which its factors' rounding to 4 bits may have moved by 2^-3.  643 us against 1030
    // for as many bf16 products.)
    __device__ __forceinline__ void mma_scaled(const xt_u4 *p, const xt_u4 *q, float f, xt_f4 &c)
    {
        const xt_f4 zero = {0, 0, 0, 0};
        xt_f4 x;
        if constexpr (T::ELEM == EXPERTS_FP8) {
            const xt_i8 xa = {(int)p[0][0], (int)p[0][1], (int)p[0][2], (int)p[0][3], (int)p[U - 1][0], (int)p[U - 1][1], (int)p[U - 1][2], (int)p[U - 1][3]};
            const xt_i8 xb = {(int)q[0][0], (int)q[0][1], (int)q[0][2], (int)q[0][3], (int)q[U - 1][0], (int)q[U - 1][1], (int)q[U - 1][2], (int)q[U - 1][3]};
            x = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xb, xa, zero, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
        } else {
            x = zero;
#pragma unroll
            for (int u = 0; u < 4; ++u) x = mma16<EXPERTS_BF16>(bf16_of(q[u / 2], u % 2), bf16_of(p[u / 2], u % 2), x);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) c[v] = __builtin_fmaf(f, x[v], c[v]);
    }

    template <int t>
    __device__ __forceinline__ void read_a(const ReadA &r, const char *la, const float *scales)
    {
        constexpr int set = t & 1, m0 = t % MSTEPS * MA;
#pragma unroll
        for (int m = 0; m < MA; ++m) {
            a[set][m][0] = r.read(la, m0 + m, T::FP8 ? 0 : t / MSTEPS);
            if constexpr (T::FP8) {
                a[set][m][U - 1] = r.read(la, m0 + m, 1);
                w[set][m] = scales[(m0 + m) * 16];
            }
        }
    }
    // the fragments of B that step t needs and the step before did not
    template <int t>
    __device__ __forceinline__ void read_b(const ReadB &r, const char *lb)
    {
        constexpr int set = B2 ? (t / MSTEPS) & 1 : 0;
        if constexpr (t % MSTEPS == 0) {
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                b[set][ni][0] = r.read(lb, ni, T::FP8 ? 0 : t / MSTEPS);
                if constexpr (T::FP8) b[set][ni][U - 1] = r.read(lb, ni, 1);
            }
        }
    }
    // the fragments of step t without the k that another stage has had
    template <int t>
    __device__ __forceinline__ void mask(const xt_u4 (&keep)[2])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const xt_u4 &w = keep[T::FP8 ? u : t / MSTEPS];
#pragma unroll
            for (int m = 0; m < MA; ++m) a[t & 1][m][u] &= w;
            if constexpr (t % MSTEPS == 0)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) b[B2 ? (t / MSTEPS) & 1 : 0][ni][u] &= w;
        }
    }
    // `hook` is called after every instruction
    template <int t, class Hook>
    __device__ __forceinline__ void mma(float wb, xt_f4 (&acc)[T::MI][T::NI], Hook hook)
    {
        constexpr int sa = t & 1, sb = B2 ? (t / MSTEPS) & 1 : 0;
#pragma unroll
        for (int m = 0; m < MA; ++m)
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                xt_f4 &c = acc[t % MSTEPS * MA + m][ni];
                const xt_u4 *p = a[sa][m], *q = b[sb][ni];
                if constexpr (!T::FP8) c = mma16<T::ELEM>(q[0], p[0], c);
                else mma_scaled(p, q, w[sa][m] * wb, c);
                hook(m * T::NI + ni);
            }
    }
};

// f(0), f(1), ... f(N - 1), the numbers known when compiled
template <int N, int I = 0, class F>
__device__ __forceinline__ void for_each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        for_each<N, I + 1>(f);
    }
}
// A constant wait: at most N of this wave's vector memory operations under way.
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
// A barrier of the workgroup; a k group of one wave needs none (and several groups of more waves meet as often as each other).
template <int NW>
__device__ __forceinline__ void meet()
{
    // (a bare s_barrier: a full fence would drain the loads under way)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if constexpr (NW > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where a wave finds the scales of its tile (fp8).
struct TileScales {
    const char *a;       // of A, k block 0 (uniform)
    uint32_t a_off;      // this lane's row, bytes
    int64_t a_step;      // bytes from block to block
    const float *b;
    int64_t b_step;
};

// The sums of a tile: acc[mi][ni] of this wave, over the k of [k0, k1) of the group; k-group waves each their stages, joined
// at the end.  True for the waves that hold the result.
//
// Stages that lie wholly inside go through the ring: S of them are requested at first, and the one barrier of a stage lies before its last
// step, when every wave has read all of it: behind it the slot is refilled with the stage S further on, and the first fragments of the
// next stage are read, which the same barrier certifies as landed.  What is left is loaded through registers, one stage at a time.
template <class T, class ARow>
__device__ __forceinline__ bool tile_sums(Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> &sa, Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> &sb,
                                          const int k0, const int k1, const int wave, const int kg, const int lane, ARow a_row, const TileScales &scales, const bool idle, xt_f4 (&acc)[T::MI][T::NI])
{
    constexpr int S = T::S, BK = T::BK, STEPS = Steps<T>::STEPS;
    constexpr int LOADS = Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE>::Q + Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false>::Q + (T::FP8 ? 1 : 0) + (T::PREFETCH ? 1 : 0);
    static_assert(S <= 5 && LOADS * (S - 1) <= 63, "the wait count is a 6-bit field");
    const int wm = wave / T::WN, wn = wave % T::WN;
    char *const ring = xt_smem + kg * (S * T::STAGE);
    const uint32_t ring_at = (uint32_t)(uintptr_t)(xt_lds_void)ring;
    Steps<T> f;
    typename Steps<T>::ReadA ra;
    typename Steps<T>::ReadB rb;
    ra.start(wm * (T::BM / T::WM), lane);
    rb.start(wn * (T::BN / T::WN), lane);
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = xt_f4{0, 0, 0, 0};

    const int k = k1 - k0;
    const int stages = k > 0 ? (k + BK - 1) / BK : 0;
    // stages that lie wholly inside both operands
    int whole = k > 0 ? k / BK : 0;
    const bool a_cut = sa.cut(), b_cut = sb.cut();
    if (a_cut) whole = stages_of_whole_units(whole, BK, k, (int64_t)sa.lines * T::ES, sa.pitch);
    if (b_cut) whole = stages_of_whole_units(whole, BK, k, (int64_t)sb.lines * T::ES, sb.pitch);
    if ((a_cut && sa.index) || (b_cut && sb.index)) whole = 0;   // (any k may name the storage's last row)
    // BACK: the k that are left are the end of one more stage, which begins before them; what it shares with the stage before is
    // masked in both operands' fragments.  (Through registers / so: fp16, 3001 x 1501 x 1003 over 7 groups
    // 35.4 / 32.4 us; 8 bits, 1777 x 1368 x 2504 over 5 36.0 / 34.5.)
    const bool back = T::BACK && whole > 0 && whole < stages && !a_cut && !b_cut;
    const int ringed = whole + (back ? 1 : 0);
    // TURN: an XCD's workgroups begin with a stage of their own and go round: rows that lie a multiple of 4 KB apart
    // have the same stage in the same memory channels, which all XCDs would ask for at once (bf16, 32768 x 4096 x 4096 over 32
    // groups as before, 16384 x 4096 x 2048 backward 691 / 672 us.  8 bits: no registers left for it; rows 4096 + 256 bytes apart, 310 / 272)
    const int turn = T::TURN ? (int)((uint32_t)whole * (blockIdx.x & 7) / 8) : 0;
    auto stage_at = [&](int s) { return T::TURN ? (s + turn < whole ? s + turn : s + turn - whole) : s; };
    auto begin_of = [&](int s) { return s < whole ? s * BK : back ? k - BK : (whole - 1) * BK; };   // (ALWAYS and BACK; past the end: the last one's)
    if constexpr (T::TURN) {
        sa.base += (int64_t)turn * BK * T::ES;
        sb.base += T::BKS ? (int64_t)turn * BK * sb.pitch : (int64_t)turn * BK * T::ES;
    }
    const int mine = ringed > kg ? (ringed - kg + T::WK - 1) / T::WK : 0;   // ... this group's
    const int plain = whole > kg ? (whole - kg + T::WK - 1) / T::WK : 0;    // ... those not moved back
    auto move_back = [&]() {   // (a branch of its own: as a part of what each request moves on by it cost the 8-bit 128 x 128 tile a third)
        sa.advance(k0 + k - BK, k - BK - whole * BK, wave, lane);
        sb.advance(k0 + k - BK, k - BK - whole * BK, wave, lane);
    };
    auto request_scales = [&](int s, int slot) {
        // (64 rows a wave; the last waves repeat others')
        dma4(scales.a + (int64_t)s * scales.a_step, scales.a_off, ring_at + (uint32_t)(slot * T::STAGE + T::A_BYTES + T::B_BYTES + (wave * 64 % (T::BM < 64 ? 64 : T::BM)) * 4));
    };
    uint32_t pre = 0;
    if constexpr (T::PREFETCH > 0)
        if (mine > 0) {   // (a group without rows: no operand need be there)
            const int at = (wave % (T::NW / 2)) * 64 + lane;
            pre = wave < T::NW / 2 ? (sa.index ? 0 : sa.line_of(at)) : (sb.index ? 0 : sb.line_of(at));
        }
    typedef Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> StagedA;
    typedef Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> StagedB;
    // instruction q of the request for this group's stage r
    auto request_one = [&](auto which, int r, int slot) {
        constexpr int q = decltype(which)::value;
        const uint32_t to = ring_at + (uint32_t)(slot * T::STAGE);
        if constexpr (q < StagedA::Q) sa.template load<q>(to, wave);
        else if constexpr (q < StagedA::Q + StagedB::Q) sb.template load<q - StagedA::Q>(to + T::A_BYTES, wave);
        if constexpr (q == StagedA::Q + StagedB::Q - 1) {
            const int s = r * T::WK + kg;
            const int at = stage_at(!T::ALWAYS || s < whole ? s : whole - 1);
            // (past the end: the last one again)
            const int ahead = T::ALWAYS && T::BACK ? begin_of(s + 1) - begin_of(s)
                              : !T::ALWAYS || s + 1 < whole ? (T::TURN && at + 1 == whole ? -at * BK : BK * T::WK) : 0;
            const int next = k0 + (T::ALWAYS && T::BACK ? begin_of(s + 1) : s * BK + ahead);
            sa.advance(next, ahead, wave, lane);
            sb.advance(next, ahead, wave, lane);
            if constexpr (T::FP8) request_scales(at, slot);
            if constexpr (T::PREFETCH > 0) {
                const int on = s + T::PREFETCH < whole ? T::PREFETCH * BK - ahead : 0;
                const bool b = wave >= T::NW / 2;
                // (rows named by an index are not known yet: the storage's first row stands for them)
                const char *const from = b ? sb.base + (sb.index ? 0 : on * sb.pitch) : sa.base + (sa.index ? 0 : on * sa.pitch);
                dma4(from, pre, ring_at + S * T::STAGE);
            }
        }
    };
    auto request = [&](int r, int slot) { for_each<StagedA::Q + StagedB::Q>([&](auto q) { request_one(q, r, slot); }); };
    auto scale_row = [&](const char *la) { return (const float *)(la + T::A_BYTES + T::B_BYTES) + wm * (T::BM / T::WM) + (lane & 15); };
    auto scale_b = [&](int s) { return T::FP8 ? scales.b[(int64_t)s * scales.b_step] : 0.0f; };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    xt_u4 keep[2];   // BACK: what stays of a lane's units
    // One stage at `la`, its first fragments read.  AFTER: read those of the stage at `after` before the last step, once `next`
    // has seen to it that they are there (known when compiled: a branch between the steps would have the compiler gather
    // the matrix instructions behind it).
    auto stage = [&](const char *la, float wb, const char *after, auto there, auto masked, auto next, auto hook) {
        constexpr bool AFTER = decltype(there)::value;
        const char *const lb = la + T::A_BYTES;
        if constexpr (Steps<T>::SPLIT) {
            // The first half of the rows a fragment at a time, the second half's being read meanwhile; then every wave has read
            // all of the stage, and the second half runs column block by column block: each of B's fragments, of which there is
            // room for one set, is done with after a quarter of it and read anew.
            constexpr int H = T::MI / 2;
            for_each<H>([&](auto t) {
                constexpr int i = decltype(t)::value;
                if constexpr (i + 1 < H) f.template read_a<i + 1>(ra, la, scale_row(la));
                f.template read_rest<i>(ra, la, scale_row(la));
                f.template mma<i>(wb, acc, [](int) {});
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (AFTER) next();
            for_each<T::NI>([&](auto n) {
                constexpr int ni = decltype(n)::value;
                for_each<H>([&](auto t) { f.mma_scaled(f.rest[decltype(t)::value], f.b[0][ni], f.rest_w[decltype(t)::value] * wb, acc[H + decltype(t)::value][ni]); });
                if constexpr (AFTER) {
                    f.read_b_one(rb, after + T::A_BYTES, ni);
                    if constexpr (ni == T::NI - 2) f.template read_a<0>(ra, after, scale_row(after));
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            return;
        }
        for_each<STEPS>([&](auto step) {
            constexpr int t = decltype(step)::value;
            if constexpr (t + 1 < STEPS) {
                f.template read_a<t + 1>(ra, la, scale_row(la));
                f.template read_b<t + 1>(rb, lb);
            } else if constexpr (AFTER) {
                next();
                if constexpr (Steps<T>::A2) f.template read_a<0>(ra, after, scale_row(after));
                if constexpr (Steps<T>::B2) f.template read_b<0>(rb, after + T::A_BYTES);
            }
            if constexpr (decltype(masked)::value) f.template mask<t>(keep);
            f.template mma<t>(wb, acc, [&](int i) { hook(step, i); });
            if constexpr (T::FP8) __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (AFTER && !Steps<T>::A2) f.template read_a<0>(ra, after, scale_row(after));
        if constexpr (AFTER && !Steps<T>::B2) f.template read_b<0>(rb, after + T::A_BYTES);
    };
    constexpr auto none = [](auto, int) {};

    // `busy`: a wave whose rows all lie past the group's end requests its part of the stages and meets the others, no more: its
    // SIMD's other wave then has the matrix cores alone
    auto run = [&](auto busy) {
    constexpr bool BUSY = decltype(busy)::value;
    if (mine > 0) {
        int slot = 0, r = 0;
        float wb = scale_b(stage_at(kg));
        auto first = [&]() {
            meet<T::NW>();
            if constexpr (BUSY) {
                f.template read_a<0>(ra, ring, scale_row(ring));
                f.template read_b<0>(rb, ring + T::A_BYTES);
            }
        };
        // stage r; `wait`: until stage r + 1 has landed; more: request the one S further on into this one's slot
        auto go = [&](auto more, auto wait) {
            const int here = slot;
            slot = slot + 1 == S ? 0 : slot + 1;
            if constexpr (!BUSY) {
                wait();
                meet<T::NW>();
                if constexpr (decltype(more)::value) request(r + S, here);
                ++r;
                return;
            }
            const float now = wb;
            wb = scale_b(stage_at((r + 1) * T::WK + kg));
            stage(ring + here * T::STAGE, now, ring + slot * T::STAGE, yes, no, [&]() {
                wait();
                meet<T::NW>();
                if constexpr (decltype(more)::value && T::SPREAD == 0) request(r + S, here);
            }, [&](auto t, int i) {
                if constexpr (decltype(more)::value && T::SPREAD > 0 && decltype(t)::value == STEPS - 1)
                    for_each<StagedA::Q + StagedB::Q>([&](auto q) { if (i == decltype(q)::value * T::SPREAD) request_one(q, r + S, here); });
            });
            ++r;
        };
        auto last = [&]() {
            // bytes of a lane's units that the stage before has had
            const int skip = back && (mine - 1) * T::WK + kg == whole ? (BK - (k - whole * BK)) * T::ES : 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int gone = skip - 64 * h - 16 * (lane >> 4) - 4 * i;
                    keep[h][i] = gone <= 0 ? ~0u : gone >= 4 ? 0u : ~0u << (8 * gone);
                }
            stage(ring + slot * T::STAGE, wb, nullptr, no, std::integral_constant<bool, T::BACK>(), []() {}, none);
        };
        auto all_but = []() { wait_vm<LOADS * (S - 2) + (T::PREFETCH ? 1 : 0)>(); };   // only the S - 2 stages behind the next may be under way
        if constexpr (T::ALWAYS) {
            // There is always a request, past the end for the last stage once more (nobody reads it there): every wait is the
            // same, and one loop does for all stages but the last.
            for (int q = 0; q < S; ++q) request(q, q);
            wait_vm<LOADS * (S - 1)>();
            first();
            while (r + 1 < mine) go(yes, all_but);
            if constexpr (BUSY) last();
        } else {
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (q < mine) {
                    if (q == plain) move_back();
                    request(q, q);
                }
            if (mine >= S) wait_vm<LOADS * (S - 1)>();
            else wait_vm<0>();
            first();
            for (int upto = plain;; upto = mine) {
                while (r + S < upto) go(yes, all_but);
                if (r + S >= mine) break;
                move_back();
            }
            while (r + 1 < mine) go(no, []() { wait_vm<0>(); });
            if constexpr (BUSY) last();
        }
    }
    if constexpr (T::ALWAYS) wait_vm<0>();   // (the requests past the end: nothing is under way when the workgroup ends)
    if constexpr (T::WK > 1 && T::NW > 1)
        for (int r = mine; r < (ringed + T::WK - 1) / T::WK; ++r) meet<T::NW>();   // (the groups that have one stage more)
    // stages that are not whole
    for (int s = ringed; s < stages; ++s) {
        if (T::WK > 1 && s % T::WK != kg) {
            if constexpr (T::NW > 1) { meet<T::NW>(); meet<T::NW>(); }
            continue;
        }
        meet<T::NW>();                 // slot 0 is no longer read
        sa.load_cut(ring, k0 + s * BK, wave, lane, a_row);
        sb.load_cut(ring + T::A_BYTES, k0 + s * BK, wave, lane, [](int i) { return i; });
        if constexpr (T::FP8) { request_scales(s, 0); wait_vm<0>(); }
        meet<T::NW>();
        if constexpr (BUSY) {
            f.template read_a<0>(ra, ring, scale_row(ring));
            f.template read_b<0>(rb, ring + T::A_BYTES);
            stage(ring, scale_b(s), nullptr, no, no, []() {}, none);
        }
    }
    };
    if (T::NW > 1 && idle) run(no);
    else run(yes);
    if constexpr (T::WK > 1) {
        // the k groups' sums, added up by the first in order (so the result does not depend on who came first)
        __syncthreads();
        constexpr int PER = T::MI * T::NI * 4 * 64;   // floats of a wave
        float *const img = (float *)xt_smem;
        if (kg > 0) {
            float *const to = img + ((kg - 1) * T::NW + wave) * PER;
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) *(xt_f4 *)(to + ((mi * T::NI + ni) * 64 + lane) * 4) = acc[mi][ni];
        }
        __syncthreads();
        if (kg > 0) return false;
#pragma unroll
        for (int g = 1; g < T::WK; ++g)
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] += *(const xt_f4 *)(img + (((g - 1) * T::NW + wave) * PER) + ((mi * T::NI + ni) * 64 + lane) * 4);
    }
    return true;
}

// Element v of acc[mi][ni] of a lane: row mi * 16 + lane % 16 of the wave's rows, column col_of(ni, lane) + v of its columns.
template <class T>
__device__ __forceinline__ int col_of(int ni, int lane)
{
    return T::PERM ? (ni >> 1) * 32 + 8 * (lane >> 4) + 4 * (ni & 1) : ni * 16 + 4 * (lane >> 4);
}
// Row blocks mi of a wave's sums into R: row i of R at element row_at(mi), columns col0 + ..., those from `from` to N - 1.  Two
// fragments at a time: a lane's columns of both are 8 in a row, as they lie (PERM) or after the odd groups of 16 lanes have
// exchanged their first fragment's for their neighbours' second's.
template <class T, class RowAt>
__device__ __forceinline__ void store_sums(const xt_f4 (&acc)[T::MI][T::NI], void *R, int out, int lane, int col0, int from, int N, RowAt row_at)
{
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) {
        const int64_t at = row_at(mi);
        if constexpr (T::NI % 2 == 0) {
#pragma unroll
            for (int ni = 0; ni < T::NI; ni += 2) {
                float x[8];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    x[v] = acc[mi][ni][v];
                    x[4 + v] = acc[mi][ni + 1][v];
                    if constexpr (!T::PERM) {
                        const auto y = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x[v]), __builtin_bit_cast(uint32_t, x[4 + v]), false, false);
                        const uint32_t lo = y[0], hi = y[1];
                        x[v] = __builtin_bit_cast(float, lo);
                        x[4 + v] = __builtin_bit_cast(float, hi);
                    }
                }
                const int c = col0 + (T::PERM ? col_of<T>(ni, lane) : ni * 16 + 16 * ((lane >> 4) & 1) + 8 * (lane >> 5));
                if (at >= 0) store_out<8>(R, out, at, c, from, N, x);
            }
        } else {
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                const float x[4] = {acc[mi][ni][0], acc[mi][ni][1], acc[mi][ni][2], acc[mi][ni][3]};
                if (at >= 0) store_out<4>(R, out, at, col0 + col_of<T>(ni, lane), from, N, x);
            }
        }
    }
}

// First line of a tile of n lines from `first` on, moved back so that it ends at the last one of an operand that is at least
// as long: lines stored across k then never end inside a unit.  (8-bit products do not: their blocks' scales are a wave's.)
__device__ __forceinline__ int inside(int first, int n, int lines)
{
    return first + n <= lines || lines < n ? first : lines - n;
}

template <class T>
__global__ void __launch_bounds__(T::NT) experts_rows_kernel(const ExpertsArgs a)
{
    static_assert(!T::AKS, "by rows: k lies along A's rows");
    static_assert(T::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kg = w / T::NW, wave = w % T::NW;
    const int tiles_n = (a.N + T::BN - 1) / T::BN;
    RowTile t;
    if (!find_row_tile<T::BM>(a, tiles_n, blockIdx.x, t)) return;
    const int row0 = t.row0 + t.tm * T::BM, from = t.tn * T::BN;   // (columns from `from` on are this tile's)
    const int col0 = T::BKS && !T::FP8 ? inside(from, T::BN, a.N) : from;
    const int wm = wave / T::WN, wn = wave % T::WN;

    xt_f4 acc[T::MI][T::NI];
    auto a_row = [&](int i) {   // storage row of row i of R; one that is not there reads row 0 and is zeros in the end
        if (!a.rows) return i;
        const int r = a.rows[i];
        return (unsigned)r < (unsigned)a.a_rows ? r : 0;
    };
    const int K = t.group < 0 ? 0 : a.K;
    Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> sa = {};
    Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> sb = {};
    const char *const B = (const char *)a.B + (int64_t)(t.group < 0 ? 0 : t.group) * a.group_b * T::ES;
    if (K > 0) {
        sa.start_kc((const char *)a.A, a.lda * T::ES, row0, t.row1, K, kg * T::BK, wave, lane, a_row, !a.rows);
        if constexpr (T::BKS) sb.start_ks(B, a.ldb * T::ES, nullptr, 0, col0, a.N, K, kg * T::BK, wave, lane);
        else sb.start_kc(B, a.ldb * T::ES, col0, a.N, K, kg * T::BK, wave, lane, [](int i) { return i; }, true);
    }
    TileScales scales = {};
    if constexpr (T::FP8) {
        const int i = row0 + (wave * 64 + lane) % (T::BM < 64 ? 64 : T::BM);
        scales.a = (const char *)a.scale_a;
        scales.a_step = a.ld_sa * 4;
        if (K > 0) scales.a_off = (uint32_t)a_row(i < t.row1 ? i : t.row1 - 1) * 4u;
        const int block = (col0 + wn * (T::BN / T::WN)) / 128, blocks = (a.N + 127) / 128;
        const int64_t at = block < blocks ? block : blocks - 1;
        scales.b = a.scale_b + (int64_t)(t.group < 0 ? 0 : t.group) * a.group_sb + (T::BKS ? at : at * a.ld_sb);
        scales.b_step = T::BKS ? a.ld_sb : 1;
    }
    if (!tile_sums<T>(sa, sb, 0, K, wave, kg, lane, a_row, scales, row0 + wm * (T::BM / T::WM) >= t.row1, acc)) return;

    if (a.rows)
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            const int i = row0 + wm * (T::BM / T::WM) + mi * 16 + (lane & 15);
            if (i < t.row1 && (unsigned)a.rows[i] >= (unsigned)a.a_rows) {
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = xt_f4{0, 0, 0, 0};
            }
        }
    store_sums<T>(acc, a.R, a.out, lane, col0 + wn * (T::BN / T::WN), from, a.N, [&](int mi) -> int64_t {
        const int i = row0 + wm * (T::BM / T::WM) + mi * 16 + (lane & 15);
        return i < t.row1 ? (int64_t)i * a.ldr : -1;
    });
}

// The weights' gradients: k runs over a group's rows, lines of A are columns of its storage, lines of B of D's.  grid: parts x tiles x groups.
// With several parts of a group's rows each writes its fp32 sums to the workspace, and experts_join_kernel adds them up in order.
template <class T>
__global__ void __launch_bounds__(T::NT) experts_sums_kernel(const ExpertsArgs a)
{
    static_assert(T::AKS && T::BKS && !T::PERM, "by sums: k runs across both storages");
    static_assert(T::LDS <= 160 * 1024 && (T::WK - 1) * T::NW * T::MI * T::NI * 1024 <= T::LDS, "LDS");
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kg = w / T::NW, wave = w % T::NW;
    const int tiles_m = (a.M + T::BM - 1) / T::BM, tiles_n = (a.N + T::BN - 1) / T::BN;
    const uint32_t tiles = (uint32_t)tiles_m * (uint32_t)tiles_n;
    // Within a group and part: panels of 8 row tiles, column by column.  An eighth of every group's tiles to each XCD where a
    // group has many (groups have unequal rows: 16384 rows over 16 groups of 2048 x 4096 450 us with an eighth of the groups to each, 396
    // so), an eighth of all tiles where it has few.
    const uint32_t xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, pieces = (uint32_t)a.G * (uint32_t)a.parts;
    uint32_t piece, in;
    if (sums_by_group(tiles)) {
        const uint32_t per = (tiles + 7) / 8;
        piece = slot / per;
        const uint32_t off = slot - piece * per, x = (xcd + piece) & 7, first = tiles * x / 8, last = tiles * (x + 1) / 8;
        if (piece >= pieces || off >= last - first) return;
        in = first + off;
    } else {
        const uint64_t all = (uint64_t)tiles * pieces;
        const uint32_t begin = (uint32_t)(all * xcd >> 3), end = (uint32_t)(all * (xcd + 1) >> 3);
        if (slot >= end - begin) return;
        piece = (begin + slot) / tiles;
        in = begin + slot - piece * tiles;
    }
    const int g = (int)(piece / (uint32_t)a.parts), part = (int)(piece - (uint32_t)g * (uint32_t)a.parts);
    int tm, tn;
    tile_in_region(in, (uint32_t)tiles_m, (uint32_t)tiles_n, tm, tn);
    const int from_m = tm * T::BM, from_n = tn * T::BN;   // (rows and columns from here on are this tile's)
    const int m0 = inside(from_m, T::BM, a.M), n0 = inside(from_n, T::BN, a.N);

    const int lo = clamp_row(a.offsets[g], a.k_rows), hi = clamp_row(a.offsets[g + 1], a.k_rows);
    const int k_all = hi > lo ? hi - lo : 0;
    // whole stages to a part
    const int chunk = ((k_all + a.parts - 1) / a.parts + T::BK - 1) / T::BK * T::BK;
    const int64_t k0 = (int64_t)part * chunk;
    const int from = k0 < k_all ? (int)k0 : k_all, to = k0 + chunk < k_all ? (int)(k0 + chunk) : k_all;

    Staged<T::BM, T::ES, T::KB, T::AKS, false, T::NW, T::WIDE> sa;
    Staged<T::BN, T::ES, T::KB, T::BKS, T::PERM, T::NW, false> sb;
    const char *const A = (const char *)a.A, *const B = (const char *)a.B;
    const int32_t *const ia = a.rows_of_b ? nullptr : a.rows, *const ib = a.rows_of_b ? a.rows : nullptr;
    sa.start_ks(ia ? A : A + (int64_t)lo * a.lda * T::ES, a.lda * T::ES, ia ? ia + lo : nullptr, a.a_rows, m0, a.M, to, from + kg * T::BK, wave, lane);
    sb.start_ks(ib ? B : B + (int64_t)lo * a.ldb * T::ES, a.ldb * T::ES, ib ? ib + lo : nullptr, a.a_rows, n0, a.N, to, from + kg * T::BK, wave, lane);
    xt_f4 acc[T::MI][T::NI];
    if (!tile_sums<T>(sa, sb, from, to, wave, kg, lane, [](int i) { return i; }, TileScales(), false, acc)) return;

    const int wm = wave / T::WN, wn = wave % T::WN;
    if (a.parts > 1) {
        float *const ws = a.workspace + ((int64_t)(g * tiles + (int64_t)tm * tiles_n + tn) * a.parts + part) * (T::BM * T::BN);
        store_sums<T>(acc, ws, EXPERTS_FP32, lane, wn * (T::BN / T::WN), 0, T::BN, [&](int mi) -> int64_t {
            return (int64_t)(wm * (T::BM / T::WM) + mi * 16 + (lane & 15)) * T::BN;
        });
        return;
    }
    store_sums<T>(acc, a.R, a.out, lane, n0 + wn * (T::BN / T::WN), from_n, a.N, [&](int mi) -> int64_t {
        const int i = m0 + wm * (T::BM / T::WM) + mi * 16 + (lane & 15);
        return i >= from_m && i < a.M ? (int64_t)g * a.group_r + (int64_t)i * a.ldr : -1;
    });
}

// (the kernel is a template argument: what it was granted is kept once for each)
template <class T, void (*kernel)(const ExpertsArgs)>
inline hipError_t launch_experts(const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    if (blocks <= 0) return hipSuccess;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    static const hipError_t granted = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
    kernel<<<dim3((unsigned)blocks), dim3(T::NT), T::LDS, s>>>(a);
    return hipGetLastError();
}

}  // namespace amulet
#endif
