// Declarations shared by the translation units of the low-rank adapters and of the gradients' norm.  Not part of the C ABI.
#ifndef AMULET_ADAPTERS_INTERNAL_H
#define AMULET_ADAPTERS_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "experts_internal.h"

namespace amulet {

// Which rows have which adapter: segments of neighbouring rows, and the adapter of each.
struct Segments {
    const int32_t *offsets;    // S + 1 first rows
    const int32_t *adapters;   // of each segment (outside 0 .. G - 1: none), or null: its own number
    int S, G, M;
};

// T[i] = scale[a] X[i] A[a]
struct DownArgs {
    Segments rows;
    const void *X, *A;
    const float *scales;       // of each adapter, or null: ones
    float *T;
    int64_t ldx, lda, group_a, ldt;
    int K, r, across;          // across: A's storage has k across its rows (K x r), else r x K
};
// (hipErrorInvalidConfiguration, before anything is launched: no launch holds it)
hipError_t launch_adapters_down(int type, const DownArgs &a, hipStream_t s);

// R[i] = X[i] W + T[i] B[a]
struct UpArgs {
    ExpertsArgs mm;            // the shared product (K = 0: none)
    Segments rows;
    const float *T;
    const void *B;
    int64_t ldt, ldb, group_b;
    int r, across;             // across: B's storage is r x N, else N x r
};
// tile: those of the products by groups, or this one: 16 x 16 with eight k groups
enum { ADAPTERS_16x16 = EXPERTS_TILES };
hipError_t launch_adapters_up_bf16(int tile, bool w_across, bool many, const UpArgs &a, int64_t blocks, hipStream_t s);
hipError_t launch_adapters_up_fp16(int tile, bool w_across, bool many, const UpArgs &a, int64_t blocks, hipStream_t s);

// R[g] = sum over the rows i of adapter g of X[i]^T T[i]
struct OuterArgs {
    Segments rows;
    const void *X;
    const float *T;
    void *R;
    float *workspace;          // fp32 sums of pieces
    int64_t ldx, ldt, ldr, group_r;
    int N, r, out, trans_r;
    int columns;               // of X to a workgroup: 128 or 64
    int quota, pieces;         // rows of a piece (0: an adapter is one), the most pieces that there can be
};
hipError_t launch_adapters_outer(int type, const OuterArgs &a, hipStream_t s);
constexpr int kOuterWaves = 4, kOuterAdapters = 1024;   // of a workgroup; the most whose rows are counted
hipError_t launch_adapters_join(const OuterArgs &a, hipStream_t s);

// The norm of several tensors' values, and the values scaled down to a largest one.  A launch has as many tensors as its
// arguments hold (4 KB: an address in 48 bits, a count in 40), in chunks of `chunk` values, kNormChunk or a few times as many, that its
// workgroups share.
enum { NORM_TENSORS = 180, NORM_BLOCKS = 2048, NORM_JOINED = 4 };
constexpr int kNormChunk = 8192;
struct NormTensors {
    uint32_t in[NORM_TENSORS], out[NORM_TENSORS];             // (out: clip only)
    uint32_t count[NORM_TENSORS];                             // values
    uint32_t first[NORM_TENSORS];                             // chunks before the tensor's
    uint16_t in_upper[NORM_TENSORS], out_upper[NORM_TENSORS];
    uint16_t more[NORM_TENSORS];                              // upper bits of the count, from bit 8 on the type
    uint32_t chunks, chunk;                                   // of all of them; values of one
    int n;
};
static_assert(sizeof(NormTensors) + 48 <= 4096, "a kernel's arguments");
struct NormArgs {
    double *sums;                       // of squares, one for each workgroup
    int n;                              // sums of all launches
    float *norm;
    float most;
    int given;                          // clip: `norm` holds the norm (else the sums are added up and the first workgroup writes it)
};
// sums[0 .. blocks - 1] of the tensors' squares
hipError_t launch_norm_sums(const NormTensors &t, double *sums, int blocks, hipStream_t s);
hipError_t launch_norm_join(const NormArgs &a, hipStream_t s);
hipError_t launch_norm_clip(const NormTensors &t, const NormArgs &a, int blocks, hipStream_t s);

}  // namespace amulet
#endif
