// The norm of all gradients of a step together, and the gradients scaled down to a largest norm.
//
// Bound by their bytes: read once for the norm, read again and written once to be clipped.  Squares are summed in fp64, where neither a
// large fp32 value's overflows nor a small one's is lost: each thread's own, then a workgroup's, in an order that the sizes fix; the
// workgroups' sums go to the workspace and are added up in order by whoever needs the norm (a workgroup of the clipping kernel each for
// itself: 8 KB from the caches in place of a launch).
#include "adapters_internal.h"
#include "experts_tile.h"

namespace amulet {

constexpr int kNormThreads = 256;

// the tensor of a chunk
__device__ __forceinline__ int tensor_of(const NormTensors &t, uint32_t chunk, int lane)
{
    int n = 0;
#pragma unroll
    for (int c = 0; c < NORM_TENSORS; c += 64) {
        const int l = c + lane;
        n += __popcll(__ballot(l < t.n && t.first[l < NORM_TENSORS ? l : 0] <= chunk));
    }
    return n - 1;
}

// V values (16 bytes) from p on as fp32
template <int TYPE>
struct Values {
    static constexpr int V = TYPE == EXPERTS_FP32 ? 4 : 8, ES = TYPE == EXPERTS_FP32 ? 4 : 2;
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
    u4 w;
    __device__ __forceinline__ void read(const char *p) { w = *(const u4 *)p; }
    __device__ __forceinline__ float value(int i) const
    {
        if constexpr (TYPE == EXPERTS_FP32) return __builtin_bit_cast(float, (uint32_t)w[i]);
        else if constexpr (TYPE == EXPERTS_BF16) return __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2]));
    }
    __device__ __forceinline__ static uint32_t pair(float lo, float hi)
    {
        if constexpr (TYPE == EXPERTS_BF16) return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16);
        else return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16);
    }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == EXPERTS_FP32) w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, (uint32_t)w[i]) * f);
            else w[i] = pair(value(2 * i) * f, value(2 * i + 1) * f);
        }
    }
    __device__ __forceinline__ void write(char *p) const { *(u4 *)p = w; }
    // single values
    __device__ __forceinline__ static float read_one(const char *p)
    {
        if constexpr (TYPE == EXPERTS_FP32) return *(const float *)p;
        else if constexpr (TYPE == EXPERTS_BF16) return __builtin_bit_cast(float, (uint32_t) * (const uint16_t *)p << 16);
        else return (float)*(const _Float16 *)p;
    }
    __device__ __forceinline__ static void write_one(char *p, float x)
    {
        if constexpr (TYPE == EXPERTS_FP32) *(float *)p = x;
        else *(uint16_t *)p = (uint16_t)pair(x, 0.0f);
    }
};

template <int TYPE>
__device__ __forceinline__ double squares_of(const char *p, int n)
{
    typedef Values<TYPE> Vs;
    constexpr int V = Vs::V, AT = 4;
    double sum = 0.0;
    int at = (int)threadIdx.x * V;
    for (; at + (AT - 1) * kNormThreads * V + V <= n; at += AT * kNormThreads * V) {
        Vs v[AT];
#pragma unroll
        for (int q = 0; q < AT; ++q) v[q].read(p + (int64_t)(at + q * kNormThreads * V) * Vs::ES);
#pragma unroll
        for (int q = 0; q < AT; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double x = v[q].value(i);
                sum = __builtin_fma(x, x, sum);
            }
    }
    for (; at < n; at += kNormThreads * V)
        for (int i = 0; i < V && at + i < n; ++i) {
            const double x = Vs::read_one(p + (int64_t)(at + i) * Vs::ES);
            sum = __builtin_fma(x, x, sum);
        }
    return sum;
}

// the sum over a workgroup, in thread 0
__device__ __forceinline__ double sum_of_block(double x)
{
    __shared__ double waves[kNormThreads / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = waves[0];
#pragma unroll
    for (int w = 1; w < kNormThreads / 64; ++w) sum += waves[w];
    return sum;
}

// f(tensor, its first value, how many) for the chunks of this workgroup
template <class F>
__device__ __forceinline__ void chunks_of_block(const NormTensors &t, F f)
{
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int x = __builtin_amdgcn_readfirstlane(tensor_of(t, c, threadIdx.x & 63));
        const int64_t from = (int64_t)(c - t.first[x]) * kNormChunk, left = t.count[x] - from;
        f(x, from, (int)(left < kNormChunk ? left : kNormChunk));
    }
}

__global__ void __launch_bounds__(kNormThreads) norm_sums_kernel(const NormTensors t, double *sums)
{
    double sum = 0.0;
    chunks_of_block(t, [&](int x, int64_t from, int n) {
        const char *const p = (const char *)t.in[x];
        switch (t.type[x]) {
        case EXPERTS_FP32: sum += squares_of<EXPERTS_FP32>(p + from * 4, n); break;
        case EXPERTS_BF16: sum += squares_of<EXPERTS_BF16>(p + from * 2, n); break;
        default: sum += squares_of<EXPERTS_FP16>(p + from * 2, n);
        }
    });
    sum = sum_of_block(sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ float norm_of(const double *sums, int n)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += kNormThreads) sum += sums[i];
    return (float)__builtin_sqrt(sum_of_block(sum));
}
__global__ void __launch_bounds__(kNormThreads) norm_join_kernel(const NormArgs a)
{
    const float norm = norm_of(a.sums, a.n);
    if (threadIdx.x == 0) *a.norm = norm;
}

template <int TYPE>
__device__ __forceinline__ void clip_values(const char *p, char *to, int n, float f)
{
    typedef Values<TYPE> Vs;
    constexpr int V = Vs::V, AT = 4;
    int at = (int)threadIdx.x * V;
    for (; at + (AT - 1) * kNormThreads * V + V <= n; at += AT * kNormThreads * V) {
        Vs v[AT];
#pragma unroll
        for (int q = 0; q < AT; ++q) v[q].read(p + (int64_t)(at + q * kNormThreads * V) * Vs::ES);
#pragma unroll
        for (int q = 0; q < AT; ++q) {
            if (f != 1.0f) v[q].scale(f);
            v[q].write(to + (int64_t)(at + q * kNormThreads * V) * Vs::ES);
        }
    }
    for (; at < n; at += kNormThreads * V)
        for (int i = 0; i < V && at + i < n; ++i) {
            const float x = Vs::read_one(p + (int64_t)(at + i) * Vs::ES);
            Vs::write_one(to + (int64_t)(at + i) * Vs::ES, f != 1.0f ? x * f : x);
        }
}

__global__ void __launch_bounds__(kNormThreads) norm_clip_kernel(const NormTensors t, const NormArgs a)
{
    float norm;
    if (a.given) norm = *a.norm;
    else {
        norm = norm_of(a.sums, a.n);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    }
    // (a norm that is no number or infinite changes nothing)
    const bool clipped = norm > a.most && norm < __builtin_inff();
    const float f = clipped ? a.most / norm : 1.0f;
    chunks_of_block(t, [&](int x, int64_t from, int n) {
        const char *const p = (const char *)t.in[x];
        char *const to = (char *)t.out[x];
        if (p == to && !clipped) return;
        switch (t.type[x]) {
        case EXPERTS_FP32: clip_values<EXPERTS_FP32>(p + from * 4, to + from * 4, n, f); break;
        case EXPERTS_BF16: clip_values<EXPERTS_BF16>(p + from * 2, to + from * 2, n, f); break;
        default: clip_values<EXPERTS_FP16>(p + from * 2, to + from * 2, n, f);
        }
    });
}

hipError_t launch_norm_sums(const NormTensors &t, double *sums, int blocks, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    norm_sums_kernel<<<dim3((unsigned)blocks), dim3(kNormThreads), 0, s>>>(t, sums);
    return hipGetLastError();
}
hipError_t launch_norm_join(const NormArgs &a, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    norm_join_kernel<<<dim3(1), dim3(kNormThreads), 0, s>>>(a);
    return hipGetLastError();
}
hipError_t launch_norm_clip(const NormTensors &t, const NormArgs &a, int blocks, hipStream_t s)
{
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    norm_clip_kernel<<<dim3((unsigned)blocks), dim3(kNormThreads), 0, s>>>(t, a);
    return hipGetLastError();
}

}  // namespace amulet
