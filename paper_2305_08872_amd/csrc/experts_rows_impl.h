// The tile shapes of the products by rows, for one operand type.
#ifndef AMULET_EXPERTS_ROWS_IMPL_H
#define AMULET_EXPERTS_ROWS_IMPL_H
#include "experts_tile.h"

namespace amulet {

template <class T>
inline hipError_t launch_experts_tile(const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    return launch_experts<T, experts_rows_kernel<T>>(a, blocks, s);
}

template <int ELEM, bool BKS>
inline hipError_t launch_experts_layout(int tile, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    switch (tile) {
    case EXPERTS_256x256:
        // (its fragments as bf16 have no room beside the accumulators)
        if constexpr (ELEM == EXPERTS_FP8_EXACT) return hipErrorInvalidValue;
        else return launch_experts_tile<ExpertTile<ELEM, 256, 256, 2, 4, 1, 2, false, BKS>>(a, blocks, s);
    case EXPERTS_128x128: return launch_experts_tile<ExpertTile<ELEM, 128, 128, 2, 2, 1, 2, false, BKS>>(a, blocks, s);
    case EXPERTS_64x128: return launch_experts_tile<ExpertTile<ELEM, 64, 128, 2, 2, 1, 3, false, BKS>>(a, blocks, s);
    case EXPERTS_64x64: return launch_experts_tile<ExpertTile<ELEM, 64, 64, 2, 2, 1, 3, false, BKS>>(a, blocks, s);
    case EXPERTS_64x64_K2: return launch_experts_tile<ExpertTile<ELEM, 64, 64, 2, 2, 2, 3, false, BKS>>(a, blocks, s);
    default: return launch_experts_tile<ExpertTile<ELEM, 16, 32, 1, 1, 4, 3, false, BKS>>(a, blocks, s);
    }
}

template <int ELEM>
inline hipError_t launch_experts_rows(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    return b_across ? launch_experts_layout<ELEM, true>(tile, a, blocks, s) : launch_experts_layout<ELEM, false>(tile, a, blocks, s);
}

}  // namespace amulet
#endif
