// The gradient of attention within a window: bfloat16, head_dim 64.
#include "sequence_bwd.h"

namespace grat {

hipError_t launch_window_bwd_bf16_d64(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream) {
    return launch_window_bwd<false, 64>(p, g, tile_rows, stream);
}

}  // namespace grat
