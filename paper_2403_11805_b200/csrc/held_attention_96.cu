// held_attention_kernel for rows of 96 channels.
#include "held_attention.cuh"

namespace llms {

template <>
int launch_held_attention<96>(int bits, int groups, int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, bool deep, cudaStream_t st)
{
    if (bits == 4 && groups == 3) return launch_held_shape<HeldShape<96, 4, 3>>(mode, a, f, item_ctas, deep, st);
    if (bits == 8 && groups == 3) return launch_held_shape<HeldShape<96, 8, 3>>(mode, a, f, item_ctas, deep, st);
    return LLMS_ERR_UNSUPPORTED;
}

}  // namespace llms
