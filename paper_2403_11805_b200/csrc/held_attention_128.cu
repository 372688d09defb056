// held_attention_kernel for rows of 128 channels.
#include "held_attention.cuh"

namespace llms {

template <>
int launch_held_attention<128>(int bits, int groups, int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, bool deep, cudaStream_t st)
{
    if (bits == 4 && groups == 1) return launch_held_shape<HeldShape<128, 4, 1>>(mode, a, f, item_ctas, deep, st);
    if (bits == 8 && groups == 1) return launch_held_shape<HeldShape<128, 8, 1>>(mode, a, f, item_ctas, deep, st);
    if (bits == 4 && groups == 2) return launch_held_shape<HeldShape<128, 4, 2>>(mode, a, f, item_ctas, deep, st);
    if (bits == 8 && groups == 2) return launch_held_shape<HeldShape<128, 8, 2>>(mode, a, f, item_ctas, deep, st);
    if (bits == 4 && groups == 4) return launch_held_shape<HeldShape<128, 4, 4>>(mode, a, f, item_ctas, deep, st);
    if (bits == 8 && groups == 4) return launch_held_shape<HeldShape<128, 8, 4>>(mode, a, f, item_ctas, deep, st);
    return LLMS_ERR_UNSUPPORTED;
}

}  // namespace llms
