// R[g] = sum over the rows i of adapter g of X[i]^T T[i]: the gradients of the adapters' matrices, N x r or r x N each.
//
// Bound by X's bytes: T and R are a few columns wide.  A workgroup has 16 F columns of X and 16 RI of T of one adapter, or of a piece of its
// rows; its waves take steps of 32 rows in turn and join their sums in LDS, in order.  A lane reads 2 F bytes of 8 rows of X
// and turns them in registers (byte permutes) into F columns of 8 rows each, the operands of F matrix instructions: lane i of 16 has
// columns F i + f in instruction f, so that what it ends with are neighbouring columns.  T is fp32 and is taken as three bf16 pieces, all
// of its bits (adapters_segments.h), X of fp16 as two.  us with the pieces' sums (5 to 7), 16384 x 4096, 4
// adapters, out of the caches, rank 16 / 32 / 64: bf16 35 / 42 / 66 (rank 16: 4.6 TB/s of X before the sums), fp16 54 / 67 / 96.
#include "adapters_segments.h"

namespace amulet {

// How an adapter's rows are shared out: pieces of about `quota` rows, an adapter without rows one too (its zeros).  Piece k of all: its
// adapter, which of how many it is.  False: there is none.  counts: the adapters' rows, of the workgroup's LDS.
struct Piece {
    int adapter, part, parts;
};
__device__ __forceinline__ void count_rows(const Segments &s, int *counts)
{
    for (int g = threadIdx.x; g < s.G; g += blockDim.x) counts[g] = 0;
    __syncthreads();
    for (int x = threadIdx.x; x < s.S; x += blockDim.x) {
        int lo, hi, g;
        segment_rows(s, x, lo, hi, g);
        if (g >= 0 && hi > lo) atomicAdd(&counts[g], hi - lo);
    }
    __syncthreads();
}
// (rows and quota together may pass 2^31)
__device__ __forceinline__ int pieces_of(int rows, int quota) { return rows > 0 ? (int)(((uint32_t)rows + (uint32_t)quota - 1) / (uint32_t)quota) : 1; }
__device__ __forceinline__ bool find_piece(const int *counts, int G, int quota, int k, int lane, Piece &p)
{
    int before = 0;
    for (int c = 0; c < G; c += 64) {
        const int n = c + lane < G ? pieces_of(counts[c + lane], quota) : 0;
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const uint64_t past = __ballot(before + sum > k);
        if (past) {
            const int l = __builtin_ctzll(past);
            p.adapter = c + l;
            p.parts = __builtin_amdgcn_readlane(n, l);
            p.part = k - (before + __builtin_amdgcn_readlane(sum, l) - p.parts);
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

template <int ELEM, int F, int RI>
__global__ void __launch_bounds__(64 * kOuterWaves) __attribute__((amdgpu_waves_per_eu(2))) adapters_outer_kernel(const OuterArgs a)
{
    constexpr int COLS = 16 * F, OF_X = ELEM == EXPERTS_FP16 ? 2 : 1;
    // the next step's operands on their way, where there are registers for them
    constexpr bool AHEAD = RI == 1 || F < 8;
    __shared__ int counts[kOuterAdapters];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 15, b = lane >> 4;
    // (The blocks of ranks of the same rows and columns lie behind one another on the same XCD, workgroups 8 apart: its cache has X then.  Rank 64, 16384
    // rows of 4096 columns, T in two pieces: 44 / 51 us, half as many reads of memory.)
    const unsigned blocks = (unsigned)((a.N + COLS - 1) / COLS), ranks = (unsigned)((a.r + 16 * RI - 1) / (16 * RI));
    const unsigned turn = blockIdx.x >> 3, at = turn / ranks * 8 + (blockIdx.x & 7), piece = at / blocks;
    if (piece >= (unsigned)a.pieces) return;
    Piece p = {(int)piece, 0, 1};
    if (a.quota > 0) {
        count_rows(a.rows, counts);
        if (!find_piece(counts, a.rows.G, a.quota, (int)piece, lane, p)) return;
    }
    const int g = p.adapter;
    // the lane's columns c0 + f, its ranks r0 + n (of T; what it ends with: ranks of line 4 b + v)
    const int c0 = (int)(at - piece * blocks) * COLS + F * i, r_block = (int)(turn % ranks) * 16 * RI, r0 = r_block + RI * i;
    // they end at X's last one
    const int col = c0 + F <= a.N || a.N < F ? c0 : a.N - F;
    const int workers = kOuterWaves * p.parts, me = p.part * kOuterWaves + wave;

    xt_f4 acc[F][RI];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int n = 0; n < RI; ++n) acc[f][n] = xt_f4{0, 0, 0, 0};

    // one step: rows base .. base + 31, of which those below `end` are there
    struct Step {
        uint32_t x[8][F / 2];
        float t[8][RI];
        int left;   // rows
    };
    // (No branch around a load, which would be waited for in it: lanes past an edge read what lies at it.  Columns and ranks that are not
    // there are sums of their own, which nobody stores; rows become zeros.)
    const int c_in = a.N < F ? 0 : col < a.N - F ? col : a.N - F;
    const bool even = a.r % RI == 0;
    int r_in[RI];
#pragma unroll
    for (int n = 0; n < RI; ++n) r_in[n] = r0 + n < a.r ? r0 + n : a.r - 1;
    const int r_even = r0 + RI <= a.r ? r0 : a.r - RI;
    // (The step's first row is an address of the wave's; rows lie less than 2^32 bytes behind it, the last one that is there at most.)
    const uint32_t x_pitch = (uint32_t)a.ldx * 2, t_pitch = (uint32_t)a.ldt * 4, x_lane = 8 * (uint32_t)b * x_pitch, t_lane = 8 * (uint32_t)b * t_pitch;
    auto load = [&](Step &s, int base, int end) {
        typedef uint32_t xs __attribute__((ext_vector_type(F / 2), aligned(2)));
        typedef float ts __attribute__((ext_vector_type(RI), aligned(4)));
        const char *const X = (const char *)a.X + (int64_t)base * x_pitch, *const T = (const char *)a.T + (int64_t)base * t_pitch;
        const uint32_t last = (uint32_t)(end - base < 32 ? end - base - 1 : 31), x_last = last * x_pitch, t_last = last * t_pitch;
        uint32_t x[8], t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t x_row = x_lane + j * x_pitch, t_row = t_lane + j * t_pitch;
            x[j] = x_row < x_last ? x_row : x_last;
            t[j] = t_row < t_last ? t_row : t_last;
        }
        if (a.N >= F) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const xs v = *(const xs *)(X + (x[j] + (uint32_t)c_in * 2));
#pragma unroll
                for (int q = 0; q < F / 2; ++q) s.x[j][q] = v[q];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const xt_u4 v = load_unit<2>(X + x[j], 0, a.N * 2);
#pragma unroll
                for (int q = 0; q < F / 2; ++q) s.x[j][q] = v[q];
            }
        }
        if (RI > 1 && even) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const ts v = *(const ts *)(T + (t[j] + (uint32_t)r_even * 4));
#pragma unroll
                for (int n = 0; n < RI; ++n) s.t[j][n] = v[n];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int n = 0; n < RI; ++n) s.t[j][n] = *(const float *)(T + (t[j] + (uint32_t)r_in[n] * 4));
        }
        s.left = end - base;
    };
    auto add = [&](Step &s) {
        if (s.left < 32)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool there = 8 * b + j < s.left;
#pragma unroll
                for (int q = 0; q < F / 2; ++q) s.x[j][q] = there ? s.x[j][q] : 0u;
#pragma unroll
                for (int n = 0; n < RI; ++n) s.t[j][n] = there ? s.t[j][n] : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int n = 0; n < RI; ++n) s.t[j][n] = whole_nan(s.t[j][n]);
        xt_u4 pt[kPieces][RI];
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int n = 0; n < RI; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) pt[p][n][q] = bf16_pair(piece_of(s.t[2 * q][n], p, kPieces), piece_of(s.t[2 * q + 1][n], p, kPieces));
#pragma unroll
        for (int f = 0; f < F; ++f) {
            // column f of the lane's 8 rows
            xt_u4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __builtin_amdgcn_perm(s.x[2 * q + 1][f / 2], s.x[2 * q][f / 2], f % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int h = 0; h < OF_X; ++h) {
                xt_u4 w = v;
                if constexpr (OF_X > 1)
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[q] = bf16_pair(piece_of(half_of<ELEM>(v[q], 0), h, 2), piece_of(half_of<ELEM>(v[q], 1), h, 2));
#pragma unroll
                for (int p = 0; p < kPieces; ++p)
#pragma unroll
                    for (int n = 0; n < RI; ++n) acc[f][n] = mma16<EXPERTS_BF16>(pt[p][n], w, acc[f][n]);
            }
        }
        sums_done();
    };

    // The wave's steps: every `workers`-th of those of the adapter's segments
    int lo = 0, hi = 0, steps = 0, s = me;   // the segment, the wave's next step of it
    int chunk = 0, l_lo = 0, l_hi = 0;
    uint64_t left = 0;
    bool started = false;
    auto next_segment = [&]() -> bool {
        if (!a.rows.adapters) {
            if (started || g >= a.rows.S) return false;
            started = true;
            int x;
            segment_rows(a.rows, g, lo, hi, x);
            lo = __builtin_amdgcn_readfirstlane(lo);
            hi = __builtin_amdgcn_readfirstlane(hi);
        } else {
            while (left == 0) {
                if (started) chunk += 64;
                started = true;
                if (chunk >= a.rows.S) return false;
                int x;
                segment_rows(a.rows, chunk + lane, l_lo, l_hi, x);
                left = __ballot(x == g && l_hi > l_lo);
            }
            const int l = __builtin_ctzll(left);
            left &= left - 1;
            lo = __builtin_amdgcn_readlane(l_lo, l);
            hi = __builtin_amdgcn_readlane(l_hi, l);
        }
        steps = hi > lo ? (hi - lo + 31) / 32 : 0;
        return true;
    };
    int base = 0, end = 0;   // the step's first row, the end of its segment
    auto next = [&](int &base) -> bool {
        while (s >= steps) {
            s -= steps;
            steps = 0;
            if (!next_segment()) return false;
        }
        base = lo + s * 32;
        end = hi;
        s += workers;
        return true;
    };
    if constexpr (AHEAD) {   // (a step past the last one reads its rows again, and is not added: no branch around a read)
        Step x, y;
        bool have = next(base);
        if (have) load(x, base, end);
        while (have) {
            const bool more = next(base);
            load(y, base, end);
            add(x);
            if (!more) break;
            have = next(base);
            load(x, base, end);
            add(y);
        }
    } else {
        Step x;
        while (next(base)) {
            load(x, base, end);
            add(x);
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
    // columns col + f (those from c0 on are the lane's own), ranks k + RI v + n: 4 RI in a row
    const bool whole = p.parts == 1;
    void *const R = whole ? a.R : (void *)a.workspace;
    const int out = whole ? a.out : EXPERTS_FP32;
    const int64_t group = whole ? (int64_t)g * a.group_r : (int64_t)piece * ((int64_t)a.N * a.r);
    const int64_t ld = whole ? a.ldr : a.trans_r ? a.N : a.r;   // (parts lie as R does)
    const int k = r_block + RI * 4 * b;
    if (!a.trans_r) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
            if (col + f < c0 || col + f >= a.N) continue;
            float v[4 * RI];
#pragma unroll
            for (int q = 0; q < 4 * RI; ++q) v[q] = acc[f][q % RI][q / RI];
#pragma unroll
            for (int q = 0; q < 4 * RI; q += 4) store_out<4>(R, out, group + (int64_t)(col + f) * ld, k + q, 0, a.r, v + q);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4 * RI; ++q) {
            float v[F];
#pragma unroll
            for (int f = 0; f < F; ++f) v[f] = acc[f][q % RI][q / RI];
            if (k + q < a.r) store_out<F>(R, out, group + (int64_t)(k + q) * ld, col, c0, a.N, v);
        }
    }
}

template <int ELEM, int F, int RI>
static hipError_t launch_outer(const OuterArgs &a, hipStream_t s)
{
    const int64_t blocks = (a.N + 16 * F - 1) / (16 * F), ranks = (a.r + 16 * RI - 1) / (16 * RI);
    const dim3 grid((unsigned)((blocks * a.pieces + 7) / 8 * 8 * ranks));
    constexpr int lds = kOuterWaves / 2 * F * RI * 1024;
    static_assert(lds + kOuterAdapters * 4 <= 64 * 1024, "LDS of an ordinary launch");
    adapters_outer_kernel<ELEM, F, RI><<<grid, dim3(64 * kOuterWaves), lds, s>>>(a);
    return hipGetLastError();
}
template <int ELEM>
static hipError_t launch_outer(const OuterArgs &a, hipStream_t s)
{
    if (a.columns == 128) return a.r <= 16 ? launch_outer<ELEM, 8, 1>(a, s) : launch_outer<ELEM, 8, 2>(a, s);
    return a.r <= 16 ? launch_outer<ELEM, 4, 1>(a, s) : launch_outer<ELEM, 4, 2>(a, s);
}
hipError_t launch_adapters_outer(int type, const OuterArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    return type == EXPERTS_BF16 ? launch_outer<EXPERTS_BF16>(a, s) : launch_outer<EXPERTS_FP16>(a, s);
}

// The pieces' sums added up in order, of adapters that have several: four neighbouring values of a matrix's line to a thread.
__global__ void __launch_bounds__(256) adapters_join_kernel(const OuterArgs a)
{
    __shared__ int counts[kOuterAdapters];
    count_rows(a.rows, counts);
    const int64_t of_group = (int64_t)a.N * a.r;
    const int lines = a.trans_r ? a.r : a.N, length = a.trans_r ? a.N : a.r, fours = (length + 3) / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, k = at / fours;
    const int c = (int)(at - k * fours) * 4, g = (int)(k / lines), line = (int)(k - (int64_t)g * lines);
    if (g >= a.rows.G) return;
    int parts = pieces_of(counts[g], a.quota);
    if (parts == 1) return;
    int first = 0;
    for (int x = 0; x < g; ++x) first += pieces_of(counts[x], a.quota);
    // (offsets that do not ascend may count rows twice: no more than the workspace has)
    first = first < a.pieces ? first : a.pieces;
    parts = first + parts <= a.pieces ? parts : a.pieces - first;
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    // (a line's last four, of which the thread's are stored)
    const int in = c + 4 <= length || length < 4 ? c : length - 4;
    const float *const from = a.workspace + (int64_t)first * of_group + (int64_t)line * length + in;
    float x[4] = {0, 0, 0, 0};
    if (length >= 4) {
        xt_f4 sum = {0, 0, 0, 0};
        int p = 0;
        for (; p + 4 <= parts; p += 4) {
            f4 y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = *(const f4 *)(from + (p + q) * of_group);
#pragma unroll
            for (int q = 0; q < 4; ++q) sum += __builtin_bit_cast(xt_f4, y[q]);
        }
        for (; p < parts; ++p) sum += __builtin_bit_cast(xt_f4, *(const f4 *)(from + p * of_group));
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = sum[v];
    } else {
        for (int p = 0; p < parts; ++p)
            for (int v = 0; v < length; ++v) x[v] += from[p * of_group + v];
    }
    store_out<4>(a.R, a.out, (int64_t)g * a.group_r + (int64_t)line * a.ldr, in, c, length, x);
}
hipError_t launch_adapters_join(const OuterArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    const int64_t threads = a.rows.G * (a.trans_r ? (int64_t)a.r * ((a.N + 3) / 4) : (int64_t)a.N * ((a.r + 3) / 4));
    adapters_join_kernel<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace amulet
