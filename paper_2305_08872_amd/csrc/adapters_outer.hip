// R[g] = sum over the rows i of adapter g of X[i]^T T[i]: the gradients of the adapters' matrices, N x r or r x N each.
//
// Bound by X's bytes: T and R are a few columns wide.  A workgroup has 128 columns of X and 16 RI of T of one adapter (and, with parts, a
// share of its rows), its eight waves take steps of 32 rows in turn and join their sums in LDS, in order.  A lane reads 16 bytes of 8
// rows of X and turns them in registers (32 byte permutes) into 8 columns of 8 rows each, the operands of 8 matrix instructions: lane
// i of 16 has columns 8 i + f in instruction f, so that what it ends with are neighbouring columns.  T is fp32 and is taken as two bf16 pieces
// for results of 16 bits, three for 32 (adapters_segments.h), X of fp16 as two.
#include "adapters_segments.h"

namespace amulet {

template <int ELEM, int RI, int PIECES>
__global__ void __launch_bounds__(64 * kOuterWaves) adapters_outer_kernel(const OuterArgs a)
{
    constexpr int F = 8, OF_X = ELEM == EXPERTS_FP16 ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, b = lane >> 4;
    const unsigned blocks = (unsigned)((a.N + kOuterColumns - 1) / kOuterColumns), piece = blockIdx.x / blocks;
    const int c0 = (int)(blockIdx.x - piece * blocks) * kOuterColumns + 8 * i, r0 = (int)blockIdx.y * 16 * RI;
    const int g = (int)(piece / (unsigned)a.parts), part = (int)(piece % (unsigned)a.parts);
    // the lane's 8 columns end at X's last one
    const int col = c0 + 8 <= a.N || a.N < 8 ? c0 : a.N - 8;
    const int workers = kOuterWaves * a.parts, me = part * kOuterWaves + wave;

    xt_f4 acc[F][RI];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int n = 0; n < RI; ++n) acc[f][n] = xt_f4{0, 0, 0, 0};

    // one step: rows base .. base + 31, of which those below `end` are there
    auto step = [&](int base, int end) {
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
        xt_u4 x[8];
        float t[RI][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = base + 8 * b + j;
            x[j] = xt_u4{0, 0, 0, 0};
            const char *const from = (const char *)a.X + (int64_t)row * a.ldx * 2;
            if (row < end && c0 < a.N) {
                if (a.N >= 8) x[j] = __builtin_bit_cast(xt_u4, *(const u4 *)(from + (int64_t)col * 2));
                else x[j] = load_unit<2>(from, 0, a.N * 2);
            }
#pragma unroll
            for (int n = 0; n < RI; ++n) {
                const int k = r0 + n * 16 + i;
                t[n][j] = row < end && k < a.r ? a.T[(int64_t)row * a.ldt + k] : 0.0f;
            }
        }
        // column f of the lane's 8 rows
        auto column = [&](int f) {
            xt_u4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __builtin_amdgcn_perm(x[2 * q + 1][f / 2], x[2 * q][f / 2], f % 2 ? 0x07060302u : 0x05040100u);
            return v;
        };
        xt_u4 pt[PIECES][RI];
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int n = 0; n < RI; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) pt[p][n][q] = bf16_pair(piece_of(t[n][2 * q], p, PIECES), piece_of(t[n][2 * q + 1], p, PIECES));
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const xt_u4 v = column(f);
#pragma unroll
            for (int h = 0; h < OF_X; ++h) {
                xt_u4 w = v;
                if constexpr (OF_X > 1)
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = bf16_pair(piece_of(half_of<ELEM>(v[q], 0), h, 2), piece_of(half_of<ELEM>(v[q], 1), h, 2));
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
#pragma unroll
                    for (int n = 0; n < RI; ++n) acc[f][n] = mma16<EXPERTS_BF16>(pt[p][n], w, acc[f][n]);
            }
        }
    };

    int done = 0;   // steps of the adapter's segments so far, modulo the workers
    auto segment = [&](int lo, int hi) {
        const int steps = (hi - lo + 31) / 32;
        int first = me - done;
        if (first < 0) first += workers;
        for (int64_t s = first; s < steps; s += workers) step(lo + (int)s * 32, hi);
        done = (int)(((int64_t)done + steps) % workers);
    };
    if (!a.rows.adapters) {
        if (g < a.rows.S) {
            int lo, hi, adapter;
            segment_rows(a.rows, g, lo, hi, adapter);
            lo = __builtin_amdgcn_readfirstlane(lo);
            hi = __builtin_amdgcn_readfirstlane(hi);
            if (hi > lo) segment(lo, hi);
        }
    } else {
        for (int c = 0; c < a.rows.S; c += 64) {
            int lo, hi, adapter;
            segment_rows(a.rows, c + lane, lo, hi, adapter);
            for (uint64_t left = __ballot(adapter == g && hi > lo); left; left &= left - 1) {
                const int l = __builtin_ctzll(left);
                segment(__builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l));
            }
        }
    }

    // the waves' sums: halves onto halves, in a fixed order
    extern __shared__ __attribute__((aligned(16))) char smem[];
    xt_f4 *const sums = (xt_f4 *)smem;
#pragma unroll
    for (int half = kOuterWaves / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int n = 0; n < RI; ++n) sums[((wave - half) * F * RI + f * RI + n) * 64 + lane] = acc[f][n];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int n = 0; n < RI; ++n) acc[f][n] += sums[(wave * F * RI + f * RI + n) * 64 + lane];
        __syncthreads();
    }
    if (wave != 0 || c0 >= a.N) return;
    // a lane's columns col + f (those from c0 on are its own), ranks r0 + 16 n + 4 b + v
    const bool whole = a.parts == 1;
    void *const R = whole ? a.R : (void *)a.workspace;
    const int out = whole ? a.out : EXPERTS_FP32;
    const int64_t group = whole ? (int64_t)g * a.group_r : ((int64_t)g * a.parts + part) * ((int64_t)a.N * a.r);
    const bool columns_first = whole && !a.trans_r;   // (parts lie r x N)
    const int64_t ld = whole ? a.ldr : a.N;
#pragma unroll
    for (int n = 0; n < RI; ++n) {
        const int k = r0 + 16 * n + 4 * b;
        if (k >= a.r) continue;
        if (columns_first) {
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const float v[4] = {acc[f][n][0], acc[f][n][1], acc[f][n][2], acc[f][n][3]};
                if (col + f >= c0 && col + f < a.N) store_out<4>(R, out, group + (int64_t)(col + f) * ld, k, 0, a.r, v);
            }
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float y[8] = {acc[0][n][v], acc[1][n][v], acc[2][n][v], acc[3][n][v], acc[4][n][v], acc[5][n][v], acc[6][n][v], acc[7][n][v]};
                if (k + v < a.r) store_out<8>(R, out, group + (int64_t)(k + v) * ld, col, c0, a.N, y);
            }
        }
    }
}

template <int ELEM, int RI>
static hipError_t launch_outer(const OuterArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)outer_blocks(a.N, a.rows.G, a.parts), (unsigned)((a.r + 16 * RI - 1) / (16 * RI)));
    constexpr int lds = kOuterWaves / 2 * 8 * RI * 1024;
    auto launch = [&](auto kernel) -> hipError_t {
        const hipError_t granted = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (granted != hipSuccess) { (void)hipGetLastError(); return granted; }
        kernel<<<grid, dim3(64 * kOuterWaves), lds, s>>>(a);
        return hipGetLastError();
    };
    return a.out == EXPERTS_FP32 ? launch(adapters_outer_kernel<ELEM, RI, 3>) : launch(adapters_outer_kernel<ELEM, RI, 2>);
}
hipError_t launch_adapters_outer(int type, const OuterArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    const bool narrow = outer_ranks(a.r) == 16;
    if (type == EXPERTS_BF16) return narrow ? launch_outer<EXPERTS_BF16, 1>(a, s) : launch_outer<EXPERTS_BF16, 2>(a, s);
    return narrow ? launch_outer<EXPERTS_FP16, 1>(a, s) : launch_outer<EXPERTS_FP16, 2>(a, s);
}

// The parts' sums added up in order: a thread to four neighbouring columns of a rank.
__global__ void __launch_bounds__(256) adapters_join_kernel(const OuterArgs a)
{
    const int64_t of_group = (int64_t)a.N * a.r;
    const int fours = (a.N + 3) / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, k = at / fours;
    const int c = (int)(at - k * fours) * 4, g = (int)(k / a.r), rank = (int)(k - (int64_t)g * a.r);
    if (g >= a.rows.G) return;
    const float *const from = a.workspace + (int64_t)g * a.parts * of_group + (int64_t)rank * a.N + c;
    float x[4] = {0, 0, 0, 0};
    for (int p = 0; p < a.parts; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (c + v < a.N) x[v] = p == 0 ? from[v] : x[v] + from[p * of_group + v];
    const int64_t group = (int64_t)g * a.group_r;
    if (a.trans_r) { store_out<4>(a.R, a.out, group + (int64_t)rank * a.ldr, c, 0, a.N, x); return; }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (c + v < a.N) {
            const float y[4] = {x[v], 0, 0, 0};
            store_out<4>(a.R, a.out, group + (int64_t)(c + v) * a.ldr, rank, 0, rank + 1, y);
        }
}
hipError_t launch_adapters_join(const OuterArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    const int64_t threads = (int64_t)a.rows.G * a.r * ((a.N + 3) / 4);
    adapters_join_kernel<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace amulet
