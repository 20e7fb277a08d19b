// A shared product with low-rank adapters, bf16 operands: the instances of adapters_up_kernel (adapters_up_impl.h).
#include "adapters_up_impl.h"

namespace amulet {

hipError_t launch_adapters_up_bf16(int tile, bool w_across, bool many, const UpArgs &a, int64_t blocks, hipStream_t s)
{
    return launch_adapters_up<EXPERTS_BF16>(tile, w_across, many, a, blocks, s);
}

}  // namespace amulet
