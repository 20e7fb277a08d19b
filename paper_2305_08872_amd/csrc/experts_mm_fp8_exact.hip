// Products by groups of rows, e4m3 operands, results of 32 bits: the instances of experts_rows_kernel (experts_tile.h).
//
// The 8-bit matrix instructions sum 128 products with what lies below some 2^-17 of the largest dropped: 1.5e-5 of a sum of normal
// values (2-norm), 3e-5 where one operand has a few large channels.  A result of 16 bits, rounded by 2e-3 or 3e-4, does not
// show it unless the large products of a block cancel.  Here the values become bf16, exactly, and the bf16 instruction sums them: 1e-8, at about half the rate (both instructions
// alone: 3922 against 1970 TFLOP/s).
#include "experts_rows_impl.h"

namespace amulet {

hipError_t launch_experts_rows_fp8_exact(int tile, bool b_across, const ExpertsArgs &a, int64_t blocks, hipStream_t s)
{
    return launch_experts_rows<EXPERTS_FP8_EXACT>(tile, b_across, a, blocks, s);
}

}  // namespace amulet
