// 8-bit floating point (e4m3) with one scale for each block of 128: scale = max(amax / 448, 2^-126), value =
// e4m3(x * (1 / scale)), to the nearest, ties to even.  448 is the type's largest value; the least scale keeps its reciprocal finite for
// blocks of zeros.  The reciprocal is rounded once per block instead of dividing every value (a value may end up on the
// other side of a tie, never further).  A NaN stays one and does not count for amax; an infinity makes its block's scale
// infinite and its own values NaN.  Bound by memory: each value is read once (16384 x 4096 bf16 by rows: 41 us = 4.95 TB/s,
// a large copy's rate).
//
// By rows (1 x 128, activations): 16 lanes have a block, 16 rows a workgroup; scales [block of columns][row], so that the
// products read those of a stage side by side.  By blocks (128 x 128, weights): a workgroup has a block, its values in registers
// (16 matrices of 4096 x 4096 bf16 147 us = 5.46 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts_internal.h"

namespace amulet {

typedef uint32_t qz_u4 __attribute__((ext_vector_type(4)));
typedef float qz_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t qz_u2 __attribute__((ext_vector_type(2)));

constexpr float QZ_MOST = 448.0f, QZ_LEAST = 0x1p-126f;

// eight neighbouring values; VEC: aligned and all there, else those below n
template <int TYPE, bool VEC>
__device__ __forceinline__ void load8(const void *p, int64_t at, int n, float (&x)[8])
{
    if constexpr (VEC) {
        if (n <= 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        } else if constexpr (TYPE == EXPERTS_FP32) {
            const qz_f4 a = *(const qz_f4 *)((const float *)p + at), b = *(const qz_f4 *)((const float *)p + at + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
        } else {
            const qz_u4 w = *(const qz_u4 *)((const uint16_t *)p + at);
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
        for (int i = 0; i < 8; ++i) {
            x[i] = 0.0f;
            if (i < n) {
                if constexpr (TYPE == EXPERTS_FP32) x[i] = ((const float *)p)[at + i];
                else if constexpr (TYPE == EXPERTS_BF16) x[i] = __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[at + i] << 16);
                else x[i] = (float)((const _Float16 *)p)[at + i];
            }
        }
    }
}

template <bool VEC>
__device__ __forceinline__ void store8(uint8_t *q, int n, const float (&x)[8], float r)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * r, x[1] * r, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * r, x[3] * r, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * r, x[5] * r, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * r, x[7] * r, hi, true);
    if constexpr (VEC) {
        if (n > 0) *(qz_u2 *)q = qz_u2{(uint32_t)lo, (uint32_t)hi};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = (uint8_t)((uint32_t)(i < 4 ? lo : hi) >> (8 * (i & 3)));
    }
}

__device__ __forceinline__ float most_of(const float (&x)[8])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
    return m;
}
// over 16 lanes
__device__ __forceinline__ float most16(float m)
{
    m = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0xB1, 0xf, 0xf, true)));
    m = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0x4E, 0xf, 0xf, true)));
    m = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0x141, 0xf, 0xf, true)));
    m = fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), 0x140, 0xf, 0xf, true)));
    return m;
}
__device__ __forceinline__ float scale_of(float most) { return fmaxf(most / QZ_MOST, QZ_LEAST); }

constexpr int QZ_BLOCKS = 4;   // blocks of a row that a lane group has under way

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantizeArgs a, const int chunks)
{
    const int in = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t row = (int64_t)(blockIdx.x / chunks) * 16 + group;
    const int kb0 = (int)(blockIdx.x % chunks) * QZ_BLOCKS, KB = (a.K + 127) / 128;
    if (row >= a.M) return;
    float x[QZ_BLOCKS][8];
#pragma unroll
    for (int b = 0; b < QZ_BLOCKS; ++b) {
        const int c = (kb0 + b) * 128 + in * 8;
        load8<TYPE, VEC>(a.X, row * a.ldx + c, a.K - c, x[b]);
    }
#pragma unroll
    for (int b = 0; b < QZ_BLOCKS; ++b) {
        if (kb0 + b >= KB) break;
        const int c = (kb0 + b) * 128 + in * 8;
        const float scale = scale_of(most16(most_of(x[b])));
        store8<VEC>(a.Q + row * a.ldq + c, a.K - c, x[b], 1.0f / scale);
        if (in == 0) a.scales[(int64_t)(kb0 + b) * a.lds + row] = scale;
    }
}

template <int TYPE, bool VEC>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const QuantizeArgs a, const int MB, const int KB)
{
    __shared__ float most[4];
    const int in = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t block = blockIdx.x;
    const int kb = (int)(block % KB), mb = (int)(block / KB % MB);
    const int64_t g = block / KB / MB;
    const int c = kb * 128 + in * 8;
    const int rows = a.M - mb * 128 < 128 ? a.M - mb * 128 : 128;
    float x[8][8], m = 0.0f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int i = p * 16 + group;
        load8<TYPE, VEC>(a.X, g * a.group_x + (int64_t)(mb * 128 + i) * a.ldx + c, i < rows ? a.K - c : 0, x[p]);
        m = fmaxf(m, most_of(x[p]));
    }
    m = most16(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
    __syncthreads();
    const float scale = scale_of(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
    const float r = 1.0f / scale;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int i = p * 16 + group;
        if (i < rows) store8<VEC>(a.Q + g * a.group_q + (int64_t)(mb * 128 + i) * a.ldq + c, a.K - c, x[p], r);
    }
    if (threadIdx.x == 0) a.scales[g * a.group_s + (int64_t)mb * a.lds + kb] = scale;
}

template <int TYPE, bool VEC>
static hipError_t launch_quantize_as(const QuantizeArgs &a, bool blocks, hipStream_t s)
{
    const int KB = (a.K + 127) / 128, MB = (a.M + 127) / 128;
    if (forced_launch_failure()) return hipErrorLaunchFailure;
    if (blocks) {
        const int64_t n = (int64_t)a.G * MB * KB;
        quantize_blocks_kernel<TYPE, VEC><<<dim3((unsigned)n), dim3(256), 0, s>>>(a, MB, KB);
    } else {
        const int chunks = (KB + QZ_BLOCKS - 1) / QZ_BLOCKS;
        const int64_t n = (int64_t)((a.M + 15) / 16) * chunks;
        quantize_rows_kernel<TYPE, VEC><<<dim3((unsigned)n), dim3(256), 0, s>>>(a, chunks);
    }
    return hipGetLastError();
}
template <int TYPE>
static hipError_t launch_quantize_type(const QuantizeArgs &a, bool blocks, hipStream_t s)
{
    const int es = TYPE == EXPERTS_FP32 ? 4 : 2;
    // eight values to a lane, 16-byte reads, 8-byte writes
    const bool vec = a.K % 8 == 0 && ((uintptr_t)a.X & 15) == 0 && a.ldx * es % 16 == 0 && a.group_x * es % 16 == 0 && ((uintptr_t)a.Q & 7) == 0 && a.ldq % 8 == 0 && a.group_q % 8 == 0;
    return vec ? launch_quantize_as<TYPE, true>(a, blocks, s) : launch_quantize_as<TYPE, false>(a, blocks, s);
}
static hipError_t launch_any(const QuantizeArgs &a, bool blocks, hipStream_t s)
{
    switch (a.type) {
    case EXPERTS_FP32: return launch_quantize_type<EXPERTS_FP32>(a, blocks, s);
    case EXPERTS_BF16: return launch_quantize_type<EXPERTS_BF16>(a, blocks, s);
    default: return launch_quantize_type<EXPERTS_FP16>(a, blocks, s);
    }
}
hipError_t launch_quantize_rows(const QuantizeArgs &a, hipStream_t s) { return launch_any(a, false, s); }
hipError_t launch_quantize_blocks(const QuantizeArgs &a, hipStream_t s) { return launch_any(a, true, s); }

}  // namespace amulet
