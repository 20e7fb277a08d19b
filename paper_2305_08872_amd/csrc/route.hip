// The router of a mixture-of-experts layer: for every token the k experts with the highest logits and their weights, and
// the rows of all (token, expert) pairs in order of expert, then of token; and its gradient.
//
// Forward: one kernel chooses (a token to L lanes, each with the logits of experts lane + L j in registers; k rounds of a
// maximum over the logits and a minimum over the indexes that have it, so that ties go to the lowest one) and counts its 64
// tokens' experts in LDS; a second one finds where each expert's rows of its tokens begin, from all counts, and ranks its
// pairs among equals by ballots, 64 to a wave.  Up to 64 tokens one workgroup does both: one launch.  Everything that decides an
// order is an integer and every sum of weights is one lane group's, so results do not depend on timing.
//
// Bounds: its bytes are few (16384 tokens x 128 experts, k = 8, fp32: 10.5 MB forward, 18 with the gradient, 2 and 4 us as a copy).  Choosing takes
// k maxima that wait for each other, 9.6 us there (10.8 by floating point maxima and an exponential in each round); placing 7.6, of
// which most is finding the bases in 256 blocks' counts; the gradient 6.4 (9.0 when it read a token's weights, then its logits).
// 8 tokens x 64 experts, k = 6: 4.5 us, one workgroup's latencies.  16 lanes to a token up to 256 experts:
// their maxima stay inside a row of lanes, without the LDS; 64 lanes for more.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "experts_internal.h"

namespace amulet {

constexpr int RT_TOKENS = 64;          // tokens that a workgroup chooses for at a time
constexpr int RT_MOST_BLOCKS = 256;    // ... workgroups: more tokens make longer blocks
constexpr int RT_MOST_EXPERTS = 1024;

static int64_t tokens_of_a_block(int64_t T)
{
    const int64_t passes = (T + (int64_t)RT_TOKENS * RT_MOST_BLOCKS - 1) / ((int64_t)RT_TOKENS * RT_MOST_BLOCKS);
    return RT_TOKENS * (passes < 1 ? 1 : passes);
}
// (one without tokens too, which writes the offsets)
int64_t route_blocks(int64_t T) { return T > 0 ? (T + tokens_of_a_block(T) - 1) / tokens_of_a_block(T) : 1; }

template <int TYPE>
__device__ __forceinline__ float load_logit(const void *p, int64_t at)
{
    if constexpr (TYPE == EXPERTS_FP32) return ((const float *)p)[at];
    else if constexpr (TYPE == EXPERTS_BF16) return __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[at] << 16);
    else return (float)((const _Float16 *)p)[at];
}

// another lane's word, by the crossbars that a group of 16 lanes has (after steps 1 and 2 the four lanes of a quad agree,
// so mirrors do for the distances 4 and 8)
template <int STEP>
__device__ __forceinline__ uint32_t of_partner(uint32_t x)
{
    if constexpr (STEP == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true);       // quad_perm 1 0 3 2
    else if constexpr (STEP == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true);  // quad_perm 2 3 0 1
    else if constexpr (STEP == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true); // row_half_mirror
    else if constexpr (STEP == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true); // row_mirror
    else return (uint32_t)__shfl_xor((int)x, STEP);
}
template <int L>
__device__ __forceinline__ uint32_t group_min(uint32_t x)
{
    x = min(x, of_partner<1>(x));
    x = min(x, of_partner<2>(x));
    x = min(x, of_partner<4>(x));
    x = min(x, of_partner<8>(x));
    if constexpr (L == 64) { x = min(x, of_partner<16>(x)); x = min(x, of_partner<32>(x)); }
    return x;
}
template <int L>
__device__ __forceinline__ float group_sum(float x)
{
    x += __builtin_bit_cast(float, of_partner<1>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, of_partner<2>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, of_partner<4>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, of_partner<8>(__builtin_bit_cast(uint32_t, x)));
    if constexpr (L == 64) { x += __shfl_xor(x, 16); x += __shfl_xor(x, 32); }
    return x;
}
template <int L>
__device__ __forceinline__ float group_max(float x)
{
    x = fmaxf(x, __builtin_bit_cast(float, of_partner<1>(__builtin_bit_cast(uint32_t, x))));
    x = fmaxf(x, __builtin_bit_cast(float, of_partner<2>(__builtin_bit_cast(uint32_t, x))));
    x = fmaxf(x, __builtin_bit_cast(float, of_partner<4>(__builtin_bit_cast(uint32_t, x))));
    x = fmaxf(x, __builtin_bit_cast(float, of_partner<8>(__builtin_bit_cast(uint32_t, x))));
    if constexpr (L == 64) { x = fmaxf(x, __shfl_xor(x, 16)); x = fmaxf(x, __shfl_xor(x, 32)); }
    return x;
}

// Logits in the order of integers, whose maxima take no canonical forms: -0 is 0, and what is never chosen (-inf, NaN) is the least.
constexpr int RT_MASKED = (int)0x807fffff;   // -inf
__device__ __forceinline__ int key_of(float x)
{
    const int bits = __builtin_bit_cast(int, x + 0.0f);
    return x > -INFINITY ? bits ^ ((bits >> 31) & 0x7fffffff) : RT_MASKED;
}
__device__ __forceinline__ float logit_of(int key) { return __builtin_bit_cast(float, key ^ ((key >> 31) & 0x7fffffff)); }
template <int L>
__device__ __forceinline__ int group_max(int x)
{
    x = max(x, (int)of_partner<1>((uint32_t)x));
    x = max(x, (int)of_partner<2>((uint32_t)x));
    x = max(x, (int)of_partner<4>((uint32_t)x));
    x = max(x, (int)of_partner<8>((uint32_t)x));
    if constexpr (L == 64) { x = max(x, (int)of_partner<16>((uint32_t)x)); x = max(x, (int)of_partner<32>((uint32_t)x)); }
    return x;
}

// a logit's share before it is divided by the sum: an infinite maximum shares among the infinite ones
__device__ __forceinline__ float term_of(float x, float most)
{
    return most == INFINITY ? (x == INFINITY ? 1.0f : 0.0f) : expf(x - most);
}

// the counts before this block and all of them, for every expert -> first row of the block's pairs in base[], offsets
// Returns the number of rows.  All threads of the workgroup.
__device__ int place_bases(const RouteArgs &a, const int32_t *counts, int blocks, int block, int *base, int *total, int *rows)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    for (int e = tid; e < a.E; e += nt) { base[e] = 0; total[e] = 0; }
    __syncthreads();
    // the blocks' rows of counts, dealt out to as many sets of E threads as there are
    const int sets = nt / a.E > 0 ? nt / a.E : 1, set = tid / a.E;
    if (set < sets)
        for (int e = sets > 1 ? tid % a.E : tid; e < a.E; e += sets > 1 ? a.E : nt) {
            int before = 0, all = 0;
#pragma unroll 16
            for (int b = sets > 1 ? set : 0; b < blocks; b += sets > 1 ? sets : 1) {
                const int n = counts[(int64_t)b * a.E + e];
                all += n;
                before += b < block ? n : 0;
            }
            atomicAdd(&base[e], before);
            atomicAdd(&total[e], all);
        }
    __syncthreads();
    if (tid < 64) {
        int sum = 0;
        for (int c = 0; c < a.E; c += 64) {
            const int n = c + tid < a.E ? total[c + tid] : 0;
            int upto = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int x = __shfl_up(upto, d);
                if (tid >= d) upto += x;
            }
            if (c + tid < a.E) {
                base[c + tid] += sum + upto - n;
                if (block == 0) a.offsets[c + tid] = sum + upto - n;
            }
            sum += __shfl(upto, 63);
        }
        if (tid == 0) {
            *rows = sum;
            if (block == 0) a.offsets[a.E] = sum;
        }
    }
    __syncthreads();
    return *rows;
}

// Rows of a block's pairs [first, last) of T x k in order, by all waves of the workgroup: 64 pairs to a wave, as many waves at a time
// as `seen` has counts of every expert for (RT_SEEN).  base[e] is the next row of expert e.
constexpr int RT_SEEN = 8192;
__device__ void place_pairs(const RouteArgs &a, const int32_t *experts, int64_t first, int64_t last, int *base, int *seen)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bits = 32 - __builtin_clz((unsigned)a.E);   // E itself stands for a dropped pair
    const int waves = RT_SEEN / a.E < 16 ? RT_SEEN / a.E : 16;
    for (int64_t p0 = first; p0 < last; p0 += 64 * waves) {
        const int64_t p = p0 + 64 * wave + lane;
        for (int i = tid; i < waves * a.E; i += 1024) seen[i] = 0;
        int e = -1;
        if (wave < waves && p < last) e = experts[p - first];
        const int key = e < 0 ? a.E : e;
        uint64_t same = ~0ull;
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((key >> b) & 1);
            same &= (key >> b) & 1 ? set : ~set;
        }
        const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        __syncthreads();
        if (e >= 0 && rank == 0) seen[wave * a.E + e] = __builtin_popcountll(same);
        __syncthreads();
        int row = -1;
        if (e >= 0) {
            row = base[e] + rank;
            for (int w = 0; w < wave; ++w) row += seen[w * a.E + e];
        }
        if (wave < waves && p < last) {
            a.place[p] = row;
            if (row >= 0) a.tokens[row] = (int32_t)(p / a.k);
        }
        if (p0 + 64 * waves >= last) break;
        __syncthreads();
        for (int x = tid; x < a.E; x += 1024)
            for (int w = 0; w < waves; ++w) base[x] += seen[w * a.E + x];
        __syncthreads();
    }
}

// L lanes to a token; V logits to a lane.  alone: the workgroup has all tokens, and places their pairs too.
template <int TYPE, int L, int V>
__global__ void __launch_bounds__(1024) route_choose_kernel(const RouteArgs a, const int block_tokens, const int alone)
{
    extern __shared__ int route_lds[];   // E counts; alone: and E bases, the number of rows, the pairs' experts, what place_pairs needs
    int *const count = route_lds;
    const int tid = threadIdx.x, lane = tid & 63;
    const int in = tid % L, group = tid / L, groups = 1024 / L;
    for (int e = tid; e < a.E; e += 1024) count[e] = 0;
    __syncthreads();
    int32_t *const chosen_lds = alone ? route_lds + 2 * a.E + 1 : nullptr;
    const int64_t t0 = (int64_t)blockIdx.x * block_tokens;
    for (int i = group; i < block_tokens; i += groups) {
        const int64_t t = t0 + i;
        if (t >= a.T) break;                              // (a whole group of lanes; the shuffles below stay within groups)
        int x[V];                                         // RT_MASKED: masked, taken or past the last expert
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = in + L * j;
            x[j] = e < a.E ? key_of(load_logit<TYPE>(a.logits, t * a.ldx + e)) : RT_MASKED;
        }
        float most = 0.0f, all = 0.0f;
        int mine = RT_MASKED, expert = -1;                // lane j: the j-th highest
        for (int j = 0; j < a.k; ++j) {
            int best = x[0];
#pragma unroll
            for (int v = 1; v < V; ++v) best = max(best, x[v]);
            best = group_max<L>(best);
            uint32_t e = 0xffffffffu;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) e = x[v] == best ? (uint32_t)(in + L * v) : e;
            e = group_min<L>(e);
            if (j == 0) {
                most = logit_of(best);
                if (!a.norm && best > RT_MASKED) {
#pragma unroll
                    for (int v = 0; v < V; ++v) all += x[v] > RT_MASKED ? term_of(logit_of(x[v]), most) : 0.0f;
                    all = group_sum<L>(all);
                }
            }
            if (in == j) { mine = best; expert = best > RT_MASKED ? (int)e : -1; }
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = e == (uint32_t)(in + L * v) ? RT_MASKED : x[v];
        }
        const float term = expert < 0 ? 0.0f : term_of(logit_of(mine), most);
        if (a.norm) all = group_sum<L>(term);
        if (in < a.k) {
            const int64_t at = t * a.k + in;
            a.experts[at] = expert;
            a.weights[at] = expert < 0 ? 0.0f : term / all;
            if (chosen_lds) chosen_lds[i * a.k + in] = expert;
            if (expert >= 0) atomicAdd(&count[expert], 1);
        }
    }
    __syncthreads();
    if (!alone) {
        for (int e = tid; e < a.E; e += 1024) a.counts[(int64_t)blockIdx.x * a.E + e] = count[e];
        return;
    }
    // all tokens are here: the counts are the totals
    int *const base = route_lds + a.E, *const rows = route_lds + 2 * a.E;
    if (tid < 64) {
        int sum = 0;
        for (int c = 0; c < a.E; c += 64) {
            const int n = c + lane < a.E ? count[c + lane] : 0;
            int upto = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            if (c + lane < a.E) {
                base[c + lane] = sum + upto - n;
                a.offsets[c + lane] = sum + upto - n;
            }
            sum += __shfl(upto, 63);
        }
        if (lane == 0) { *rows = sum; a.offsets[a.E] = sum; }
    }
    __syncthreads();
    const int64_t pairs = (int64_t)a.T * a.k;
    place_pairs(a, chosen_lds, 0, pairs, base, chosen_lds + RT_TOKENS * a.k);
    for (int64_t r = *rows + tid; r < pairs; r += 1024) a.tokens[r] = -1;
}

__global__ void __launch_bounds__(1024) route_place_kernel(const RouteArgs a, const int block_tokens)
{
    extern __shared__ int route_lds[];   // E bases, E totals, the number of rows, what place_pairs needs
    const int rows = place_bases(a, a.counts, gridDim.x, blockIdx.x, route_lds, route_lds + a.E, route_lds + 2 * a.E);
    const int64_t pairs = (int64_t)a.T * a.k;
    const int64_t first = (int64_t)blockIdx.x * block_tokens * a.k;
    const int64_t last = first + (int64_t)block_tokens * a.k < pairs ? first + (int64_t)block_tokens * a.k : pairs;
    place_pairs(a, a.experts + first, first, last, route_lds, route_lds + 2 * a.E + 1);
    // rows that no pair has
    for (int64_t r = rows + (int64_t)blockIdx.x * 1024 + threadIdx.x; r < pairs; r += (int64_t)gridDim.x * 1024) a.tokens[r] = -1;
}

// dx = p (up - sum p up), up: the weights' gradients at the chosen experts; p: the weights (norm) or the softmax over all.
// A token to L lanes, each with the logits of experts lane + L j and one of the chosen ones, all asked for at once; the row passes through LDS, where
// the chosen experts' parts are added (each expert once: no two lanes meet).
template <int TYPE, int L, int V>
__global__ void __launch_bounds__(256) route_grad_kernel(const RouteArgs a)
{
    extern __shared__ float grad_lds[];
    const int in = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t t = (int64_t)blockIdx.x * (256 / L) + group;
    if (t >= a.T) return;
    float *const row = grad_lds + group * a.E;
    int e = -1;
    float w = 0.0f, up = 0.0f;
    if (in < a.k) {
        e = a.experts[t * a.k + in];
        w = a.weights[t * a.k + in];
        up = a.dweights[t * a.k + in];
    }
    float x[V];
    if (!a.norm) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = in + L * v < a.E ? load_logit<TYPE>(a.logits, t * a.ldx + in + L * v) : -INFINITY;
    }
    if ((unsigned)e >= (unsigned)a.E) { e = -1; w = 0.0f; up = 0.0f; }
    const float mean = group_sum<L>(w * up);
    if (a.norm) {
        for (int i = in; i < a.E; i += L) row[i] = 0.0f;
    } else {
        float most = -INFINITY, all = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = x[v] > -INFINITY ? x[v] : -INFINITY;    // (NaN: masked)
            most = fmaxf(most, x[v]);
        }
        most = group_max<L>(most);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = x[v] > -INFINITY ? term_of(x[v], most) : 0.0f;
            all += x[v];
        }
        all = group_sum<L>(all);
        const float scale = all > 0.0f ? -mean / all : 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (in + L * v < a.E) row[in + L * v] = x[v] > 0.0f ? x[v] * scale : 0.0f;   // (masked: whatever the mean is)
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (e >= 0) row[e] += a.norm ? w * (up - mean) : w * up;
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    for (int i = in; i < a.E; i += L) {
        const int64_t at = t * a.lddx + i;
        if constexpr (TYPE == EXPERTS_FP32) ((float *)a.dlogits)[at] = row[i];
        else if constexpr (TYPE == EXPERTS_BF16) ((__bf16 *)a.dlogits)[at] = (__bf16)row[i];
        else ((_Float16 *)a.dlogits)[at] = (_Float16)row[i];
    }
}

template <int TYPE, int L, int V>
static hipError_t launch_choose(const RouteArgs &a, hipStream_t s)
{
    const int64_t block_tokens = tokens_of_a_block(a.T), blocks = route_blocks(a.T);
    const bool alone = blocks == 1 && block_tokens == RT_TOKENS;
    const size_t seen = (RT_SEEN / a.E < 16 ? RT_SEEN / a.E : 16) * (size_t)a.E;
    const size_t lds = alone ? (2 * (size_t)a.E + 1 + RT_TOKENS * (size_t)a.k + seen) * 4 : (size_t)a.E * 4;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    route_choose_kernel<TYPE, L, V><<<dim3((unsigned)blocks), dim3(1024), lds, s>>>(a, (int)block_tokens, alone ? 1 : 0);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || alone) return e;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    route_place_kernel<<<dim3((unsigned)blocks), dim3(1024), (2 * (size_t)a.E + 1 + seen) * 4, s>>>(a, (int)block_tokens);
    return hipGetLastError();
}
template <int TYPE>
static hipError_t launch_route_type(const RouteArgs &a, hipStream_t s)
{
    if (a.k <= 16) {
        if (a.E <= 64) return launch_choose<TYPE, 16, 4>(a, s);
        if (a.E <= 128) return launch_choose<TYPE, 16, 8>(a, s);
        if (a.E <= 256) return launch_choose<TYPE, 16, 16>(a, s);
    }
    return launch_choose<TYPE, 64, 16>(a, s);
}
hipError_t launch_route(const RouteArgs &a, hipStream_t s)
{
    switch (a.type) {
    case EXPERTS_FP32: return launch_route_type<EXPERTS_FP32>(a, s);
    case EXPERTS_BF16: return launch_route_type<EXPERTS_BF16>(a, s);
    default: return launch_route_type<EXPERTS_FP16>(a, s);
    }
}

template <int TYPE>
static hipError_t launch_grad_type(const RouteArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    const dim3 small((unsigned)((a.T + 15) / 16)), large((unsigned)((a.T + 3) / 4));
    const size_t row = (size_t)a.E * 4;
    if (route_grad_lanes(a.E, a.k) == 64) route_grad_kernel<TYPE, 64, 16><<<large, dim3(256), 4 * row, s>>>(a);
    else if (a.E <= 64) route_grad_kernel<TYPE, 16, 4><<<small, dim3(256), 16 * row, s>>>(a);
    else if (a.E <= 128) route_grad_kernel<TYPE, 16, 8><<<small, dim3(256), 16 * row, s>>>(a);
    else route_grad_kernel<TYPE, 16, 16><<<small, dim3(256), 16 * row, s>>>(a);
    return hipGetLastError();
}
hipError_t launch_route_grad(const RouteArgs &a, hipStream_t s)
{
    switch (a.type) {
    case EXPERTS_FP32: return launch_grad_type<EXPERTS_FP32>(a, s);
    case EXPERTS_BF16: return launch_grad_type<EXPERTS_BF16>(a, s);
    default: return launch_grad_type<EXPERTS_FP16>(a, s);
    }
}

}  // namespace amulet
