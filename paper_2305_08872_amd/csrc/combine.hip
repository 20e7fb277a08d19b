// The experts' rows back to their tokens, R[t] = sum_j w[t][j] Y[place[t][j]], and the gradients of both factors.
// Bound by memory: every row of Y is read once.  Forward: a wave has 512 (32 bits: 256) columns of a token, its places and
// weights in scalar registers.  Backward: a wave has one (token, expert) pair, whose dot product it sums alone.
// 16384 tokens of 2048 bf16, k = 8, one pair in 50 dropped: forward 137 us (4.3 TB/s of the 4.95 of a large copy), backward 215 (5.1; each row of the
// sum's gradient is read once from memory and seven times from L2); 8 tokens of 4096, k = 6: 3.7 us, a launch's latency.
// Sums in fp32, in the order of j, rounded once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts_internal.h"

namespace amulet {

typedef float cb_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t cb_u4 __attribute__((ext_vector_type(4)));

template <int TYPE>
struct Row16 {   // 16 bytes of a row
    static constexpr int ES = TYPE == EXPERTS_FP32 ? 4 : 2, V = 16 / ES;
    static __device__ __forceinline__ float one(const void *p, int64_t at)
    {
        if constexpr (TYPE == EXPERTS_FP32) return ((const float *)p)[at];
        else if constexpr (TYPE == EXPERTS_BF16) return __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[at] << 16);
        else return (float)((const _Float16 *)p)[at];
    }
    // VEC: whole and aligned; else the values below `n`
    template <bool VEC>
    static __device__ __forceinline__ void load(const void *p, int64_t at, int n, float (&x)[V])
    {
        if constexpr (VEC) {
            if constexpr (TYPE == EXPERTS_FP32) {
                const cb_f4 v = *(const cb_f4 *)((const float *)p + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = v[i];
            } else {
                const cb_u4 w = *(const cb_u4 *)((const char *)p + at * ES);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (TYPE == EXPERTS_BF16) {
                        x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
                        x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
                    } else {
                        x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
                        x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = i < n ? one(p, at + i) : 0.0f;
        }
    }
    // rounded once, to the rows' type
    template <bool VEC>
    static __device__ __forceinline__ void store(void *p, int64_t at, int n, const float (&x)[V])
    {
        if constexpr (TYPE == EXPERTS_FP32) {
            float *const q = (float *)p + at;
            if constexpr (VEC) *(cb_f4 *)q = cb_f4{x[0], x[1], x[2], x[3]};
            else
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < n) q[i] = x[i];
        } else {
            uint16_t h[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (TYPE == EXPERTS_BF16) h[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
                else h[i] = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
            }
            uint16_t *const q = (uint16_t *)p + at;
            if constexpr (VEC) {
                cb_u4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | ((uint32_t)h[2 * i + 1] << 16);
                *(cb_u4 *)q = w;
            } else
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < n) q[i] = h[i];
        }
    }
};

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs a, const int chunks, const int64_t items)
{
    typedef Row16<TYPE> X;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t t = item / chunks;
    const int c = (int)(item % chunks) * (64 * X::V) + (threadIdx.x & 63) * X::V;
    if (c >= a.H) return;
    const int32_t *const place = a.place + t * a.k;
    const float *const w = a.weights ? a.weights + t * a.k : nullptr;
    float sum[X::V] = {};
#pragma unroll 4
    for (int j = 0; j < a.k; ++j) {
        const int row = place[j];
        if ((uint64_t)(int64_t)row >= (uint64_t)a.rows) continue;   // (dropped)
        const float f = w ? w[j] : 1.0f;
        float y[X::V];
        X::template load<VEC>(a.Y, (int64_t)row * a.ldy + c, a.H - c, y);
#pragma unroll
        for (int i = 0; i < X::V; ++i) sum[i] = __builtin_fmaf(f, y[i], sum[i]);
    }
    X::template store<VEC>(a.R, t * a.ldr + c, a.H - c, sum);
}

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256) combine_grad_kernel(const CombineArgs a, const int64_t items)
{
    typedef Row16<TYPE> X;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (item >= items) return;
    const int lane = threadIdx.x & 63;
    const int row = a.place[item];
    const bool there = (uint64_t)(int64_t)row < (uint64_t)a.rows;
    float dot = 0.0f;
    if (there) {
        const int64_t t = item / a.k;
        const float f = a.weights ? a.weights[item] : 1.0f;
#pragma unroll 4
        for (int c = lane * X::V; c < a.H; c += 64 * X::V) {
            float d[X::V], y[X::V];
            X::template load<VEC>(a.R, t * a.ldr + c, a.H - c, d);
            if (a.dweights) {
                X::template load<VEC>(a.Y, (int64_t)row * a.ldy + c, a.H - c, y);
#pragma unroll
                for (int i = 0; i < X::V; ++i) dot = __builtin_fmaf(d[i], y[i], dot);
            }
#pragma unroll
            for (int i = 0; i < X::V; ++i) d[i] *= f;
            X::template store<VEC>(a.dY, (int64_t)row * a.lddy + c, a.H - c, d);
        }
    }
    if (!a.dweights) return;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) dot += __shfl_xor(dot, s);
    if (lane == 0) a.dweights[item] = dot;
}

static bool rows16(const void *p, int64_t ld, int es) { return ((uintptr_t)p & 15) == 0 && ld * es % 16 == 0; }

template <int TYPE, bool VEC>
static hipError_t launch_combine_as(const CombineArgs &a, bool grad, hipStream_t s)
{
    const int per = 64 * Row16<TYPE>::V, chunks = (a.H + per - 1) / per;
    const int64_t items = grad ? (int64_t)a.T * a.k : (int64_t)a.T * chunks;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    const dim3 grid((unsigned)((items + 3) / 4));
    if (grad) combine_grad_kernel<TYPE, VEC><<<grid, dim3(256), 0, s>>>(a, items);
    else combine_kernel<TYPE, VEC><<<grid, dim3(256), 0, s>>>(a, chunks, items);
    return hipGetLastError();
}
template <int TYPE>
static hipError_t launch_combine_type(const CombineArgs &a, bool grad, hipStream_t s)
{
    const int es = Row16<TYPE>::ES;
    const bool vec = a.H * es % 16 == 0 && rows16(a.R, a.ldr, es) && ((grad && !a.dweights) || rows16(a.Y, a.ldy, es)) && (!grad || rows16(a.dY, a.lddy, es));
    return vec ? launch_combine_as<TYPE, true>(a, grad, s) : launch_combine_as<TYPE, false>(a, grad, s);
}
static hipError_t launch_any(const CombineArgs &a, bool grad, hipStream_t s)
{
    switch (a.type) {
    case EXPERTS_FP32: return launch_combine_type<EXPERTS_FP32>(a, grad, s);
    case EXPERTS_BF16: return launch_combine_type<EXPERTS_BF16>(a, grad, s);
    default: return launch_combine_type<EXPERTS_FP16>(a, grad, s);
    }
}
hipError_t launch_combine(const CombineArgs &a, hipStream_t s) { return launch_any(a, false, s); }
hipError_t launch_combine_grad(const CombineArgs &a, hipStream_t s) { return launch_any(a, true, s); }

}  // namespace amulet
