// Products by groups of rows, bf16 operands: the instances of experts_rows_kernel (experts_tile.h).
#include "experts_rows_impl.h"

namespace amulet {

hipError_t launch_experts_rows_bf16(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    return launch_experts_rows<EXPERTS_BF16>(tile, b_across, a, blocks, s);
}

}  // namespace amulet
