// The norm of all gradients of a step together, and the gradients scaled down to a largest norm.
//
// Bound by their bytes: read once for the norm, read again and written once to be clipped.  Squares are summed in fp64, where neither a
// large fp32 value's overflows nor a small one's is lost: each thread's own, then a workgroup's, in an order that the sizes fix; the
// workgroups' sums go to the workspace and are added up in order by whoever needs the norm (a workgroup of the clipping kernel each for
// itself: up to 64 KB from the caches, 8 or 16 as a rule, in place of a launch).  us: the norm of 2^28 bf16 values 97 (5.5 TB/s), 2^29 clipped, from the last to the first, which the
// caches may still have, 579 (3.2 GB of reads and writes at a copy's rate: 633).
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
    __device__ __forceinline__ void write(char *p) const { __builtin_nontemporal_store(w, (u4 *)p); }
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

// 4096 values, read by a workgroup at a time
constexpr int kNormBatch = 4096;
template <int TYPE>
struct Batch {
    typedef Values<TYPE> Vs;
    static constexpr int AT = kNormBatch / kNormThreads / Vs::V, STEP = kNormThreads * Vs::V;
    Vs v[AT];
    __device__ __forceinline__ void read(const char *p, int n)   // batch n
    {
#pragma unroll
        for (int q = 0; q < AT; ++q) v[q].read(p + (int64_t)(n * kNormBatch + (int)threadIdx.x * Vs::V + q * STEP) * Vs::ES);
    }
};
// all(batch, its number) for the whole batches of n values, the next one on its way; some(first value) for 16 bytes of a thread, one(value) for what is left
template <int TYPE, class All, class Some, class One>
__device__ __forceinline__ void over_values(const char *p, int n, All all, Some some, One one)
{
    typedef Batch<TYPE> B;
    const int batches = n / kNormBatch;
    if (batches > 0) {
        // (past the last one it is read again: no branch around a read)
        B x, y;
        x.read(p, 0);
        for (int i = 0;; i += 2) {
            y.read(p, i + 1 < batches ? i + 1 : batches - 1);
            all(x, i);
            if (i + 1 >= batches) break;
            x.read(p, i + 2 < batches ? i + 2 : batches - 1);
            all(y, i + 1);
            if (i + 2 >= batches) break;
        }
    }
    int at = batches * kNormBatch + (int)threadIdx.x * Values<TYPE>::V;
    for (; at + Values<TYPE>::V <= n; at += B::STEP) some(at);
    for (int i = at; i < n; ++i) one(i);
}

template <int TYPE>
__device__ __forceinline__ double squares_of(const char *p, int n)
{
    typedef Values<TYPE> Vs;
    double sum = 0.0;
    auto add = [&](const Vs &v) {
#pragma unroll
        for (int i = 0; i < Vs::V; ++i) {
            const double x = v.value(i);
            sum = __builtin_fma(x, x, sum);
        }
    };
    over_values<TYPE>(p, n,
        [&](const Batch<TYPE> &b, int) {
#pragma unroll
            for (int q = 0; q < Batch<TYPE>::AT; ++q) add(b.v[q]);
        },
        [&](int at) {
            Vs v;
            v.read(p + (int64_t)at * Vs::ES);
            add(v);
        },
        [&](int i) {
            const double x = Vs::read_one(p + (int64_t)i * Vs::ES);
            sum = __builtin_fma(x, x, sum);
        });
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

// Chunk c: its tensor's type, addresses of its values, how many they are.  BACK: each tensor's chunks from the last one on.
struct Chunk {
    const char *in;
    char *out;
    int n, type;
};
template <bool BACK>
__device__ __forceinline__ Chunk chunk_of(const NormTensors &t, uint32_t c)
{
    const int x = __builtin_amdgcn_readfirstlane(tensor_of(t, c, threadIdx.x & 63));
    const int64_t count = ((int64_t)(t.more[x] & 255) << 32) | t.count[x], chunks = (count + t.chunk - 1) / t.chunk;
    const int64_t at = c - t.first[x], from = (BACK ? chunks - 1 - at : at) * (int64_t)t.chunk, left = count - from;
    Chunk y;
    y.type = t.more[x] >> 8;
    const int64_t bytes = from * (y.type == EXPERTS_FP32 ? 4 : 2);
    y.in = (const char *)(((uint64_t)t.in_upper[x] << 32) | t.in[x]) + bytes;
    y.out = (char *)(((uint64_t)t.out_upper[x] << 32) | t.out[x]) + bytes;
    y.n = (int)(left < (int64_t)t.chunk ? left : (int64_t)t.chunk);
    return y;
}

__global__ void __launch_bounds__(kNormThreads) norm_sums_kernel(const NormTensors t, double *sums)
{
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Chunk x = chunk_of<false>(t, c);
        switch (x.type) {
        case EXPERTS_FP32: sum += squares_of<EXPERTS_FP32>(x.in, x.n); break;
        case EXPERTS_BF16: sum += squares_of<EXPERTS_BF16>(x.in, x.n); break;
        default: sum += squares_of<EXPERTS_FP16>(x.in, x.n);
        }
    }
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
__device__ __forceinline__ void clip_values(const Chunk &c, float f)
{
    typedef Values<TYPE> Vs;
    over_values<TYPE>(c.in, c.n,
        [&](Batch<TYPE> &b, int n) {
#pragma unroll
            for (int q = 0; q < Batch<TYPE>::AT; ++q) {
                if (f != 1.0f) b.v[q].scale(f);
                b.v[q].write(c.out + (int64_t)(n * kNormBatch + (int)threadIdx.x * Vs::V + q * Batch<TYPE>::STEP) * Vs::ES);
            }
        },
        [&](int at) {
            Vs v;
            v.read(c.in + (int64_t)at * Vs::ES);
            if (f != 1.0f) v.scale(f);
            v.write(c.out + (int64_t)at * Vs::ES);
        },
        [&](int i) {
            const float x = Vs::read_one(c.in + (int64_t)i * Vs::ES);
            Vs::write_one(c.out + (int64_t)i * Vs::ES, f != 1.0f ? x * f : x);
        });
}

// The chunks in the order opposite to the sums': what those read last is still in the caches.
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
    for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const Chunk x = chunk_of<true>(t, c);
        if (x.in == x.out && !clipped) continue;
        switch (x.type) {
        case EXPERTS_FP32: clip_values<EXPERTS_FP32>(x, f); break;
        case EXPERTS_BF16: clip_values<EXPERTS_BF16>(x, f); break;
        default: clip_values<EXPERTS_FP16>(x, f);
        }
    }
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
