// The weights' gradients of products by groups of rows: the instances of experts_sums_kernel (experts_tile.h), and the sum of
// the parts that a group's rows were summed in.
//
// dB[g] = sum over g's rows of A^T D: both operands lie across k, so both are read by ds_read_b64_tr_b16.  Bound by the matrix cores
// and, more than the products by rows, by each tile's start: a group's sum is short (16384 rows over 16 groups of 2048 x
// 4096, some 16 stages of 64 rows to a tile: 345 us = 797 TFLOP/s; the same rows in 4 groups, 64 stages, 262 = 1050).  A round of tiles writes
// what memory takes 7 us for, while no tile computes.
// Rows of A gathered by an index: 64-bit addresses from an index that is read a stage ahead, and no lines asked for ahead of it (the
// same sum from 4096 rows that 16384 name 413 to 420 us, where A's rows in order take 340 to 346).
// Few outputs and many rows: parts of a group's rows on more of the chip, their fp32 tiles added up in order.
#include "experts_tile.h"

namespace amulet {

template <int ELEM>
static hipError_t launch_sums(int tile, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    typedef ExpertTile<ELEM, 256, 256, 2, 4, 1, 2, true, true> Large;
    typedef ExpertTile<ELEM, 128, 128, 2, 2, 1, 2, true, true> Middle;
    typedef ExpertTile<ELEM, 64, 64, 2, 2, 1, 3, true, true> Small;
    if (tile == EXPERTS_256x256) return launch_experts<Large, experts_sums_kernel<Large>>(a, blocks, s);
    if (tile == EXPERTS_128x128) return launch_experts<Middle, experts_sums_kernel<Middle>>(a, blocks, s);
    return launch_experts<Small, experts_sums_kernel<Small>>(a, blocks, s);
}

hipError_t launch_experts_sums(int type, int tile, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    return type == EXPERTS_BF16 ? launch_sums<EXPERTS_BF16>(tile, a, blocks, s) : launch_sums<EXPERTS_FP16>(tile, a, blocks, s);
}

// One workgroup to 1024 outputs of a tile, four neighbouring ones to a lane: the parts' tiles lie one behind the other.
__global__ void __launch_bounds__(256) experts_join_kernel(const ExpertsArgs a, const int bm, const int bn)
{
    const int tiles_m = (a.M + bm - 1) / bm, tiles_n = (a.N + bn - 1) / bn, per = bm * bn / 1024;
    const int64_t tile = blockIdx.x / per;
    const int at = (int)(blockIdx.x % per) * 1024 + (int)threadIdx.x * 4;
    const int64_t tiles = (int64_t)tiles_m * tiles_n;
    const int g = (int)(tile / tiles), in = (int)(tile % tiles);
    // (tiles at the edge are moved back: experts_sums_kernel)
    const int from_m = in / tiles_n * bm, from_n = in % tiles_n * bn;
    const int i = inside(from_m, bm, a.M) + at / bn, c = inside(from_n, bn, a.N) + at % bn;
    if (i < from_m || i >= a.M) return;
    const float *ws = a.workspace + tile * a.parts * (int64_t)(bm * bn) + at;
    xt_f4 sum = *(const xt_f4 *)ws;
    for (int p = 1; p < a.parts; ++p) sum += *(const xt_f4 *)(ws + (int64_t)p * bm * bn);
    const float x[4] = {sum[0], sum[1], sum[2], sum[3]};
    store_out<4>(a.R, a.out, (int64_t)g * a.group_r + (int64_t)i * a.ldr, c, from_n, a.N, x);
}

hipError_t launch_experts_join(int tile, const ExpertsArgs &a, hipStream_t s)
{
    const int bm = kExpertsTileRows[tile], bn = kExpertsTileCols[tile];
    const int64_t tiles = (int64_t)((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn) * a.G;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    experts_join_kernel<<<dim3((unsigned)(tiles * (bm * bn / 1024))), dim3(256), 0, s>>>(a, bm, bn);
    return hipGetLastError();
}

}  // namespace amulet
