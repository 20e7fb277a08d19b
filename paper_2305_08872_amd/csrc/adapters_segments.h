// What the kernels of the low-rank adapters share: segments of rows, and fp32 values as sums of bf16 ones.
#ifndef AMULET_ADAPTERS_SEGMENTS_H
#define AMULET_ADAPTERS_SEGMENTS_H

#include "adapters_internal.h"
#include "experts_tile.h"

namespace amulet {

// The last of a segment's first rows that is not behind `row` (0 where all are): a wave looks at 64 of them at a time.  (Offsets that do
// not ascend give some number of 0 .. S.)
__device__ __forceinline__ int segment_of(const Segments &g, int row, int lane)
{
    int at = 0;
    for (int range = g.S + 1; range > 1;) {
        const int step = (range + 63) / 64;
        const int64_t s = at + (int64_t)lane * step;
        const uint64_t before = __ballot(s <= g.S && clamp_row(g.offsets[s <= g.S ? s : g.S], g.M) <= row);
        const int n = __popcll(before);
        at += n > 0 ? (n - 1) * step : 0;
        range = step;
        if (at > g.S) at = g.S;
    }
    return at;
}
// Rows and adapter of segment s (of each lane); an adapter below 0: none, or no such segment
__device__ __forceinline__ void segment_rows(const Segments &g, int s, int &lo, int &hi, int &adapter)
{
    lo = hi = 0;
    adapter = -1;
    if (s < 0 || s >= g.S) return;
    lo = clamp_row(g.offsets[s], g.M);
    hi = clamp_row(g.offsets[s + 1], g.M);
    const int x = g.adapters ? g.adapters[s] : s;
    adapter = (unsigned)x < (unsigned)g.G ? x : -1;
}

// An fp32 value as a sum of bf16 ones: the first has the sign and the upper 8 bits (no rounding: it does not become infinite), the next
// what is left.  Two keep 16 bits (all that an fp16 value has), three all 24.  A piece of which nothing is left (or of an infinity) is the one before times
// 2^-30, far below the sum's rounding, so that a product with an infinity has its sign in every piece and is no NaN; zeros stay zeros.  (What of a value lies
// below bf16's smallest, 2^-133, is lost: bits of values below 2^-109; a piece of one below 2^-103 may be zero, and a product of that with an infinity NaN.)
constexpr int kPieces = 3;   // of T's values
__device__ __forceinline__ float piece_first(float x)
{
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
}
__device__ __forceinline__ float piece_rest(float x, float first)
{
    const float rest = x - first;
    return __builtin_fabsf(rest) > 0.0f ? rest : first * 0x1p-30f;
}
// piece `which` of `pieces` (2 or 3).  (Of a NaN whose upper 7 bits of payload are zeros, which no operation makes, the first would be an infinity: a
// caller's values pass through whole_nan().)
__device__ __forceinline__ float piece_of(float x, int which, int pieces)
{
    const float p0 = piece_first(x), r1 = piece_rest(x, p0);
    const float p1 = pieces > 2 ? piece_first(r1) : r1, r2 = piece_rest(r1, p1);
    return which == 0 ? p0 : which == 1 ? p1 : r2;
}
__device__ __forceinline__ float whole_nan(float x) { return x != x ? __builtin_nanf("") : x; }
// two values rounded to bf16 side by side
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16);
}
// both 16-bit halves as fp32
template <int ELEM>
__device__ __forceinline__ float half_of(uint32_t w, int h)
{
    if constexpr (ELEM == EXPERTS_BF16) return __builtin_bit_cast(float, h ? w & 0xffff0000u : w << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(h ? w >> 16 : w));
}

}  // namespace amulet
#endif
