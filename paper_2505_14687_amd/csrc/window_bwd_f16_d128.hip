// The gradient of attention within a window: half, head_dim 128.
#include "sequence_bwd.h"

namespace grat {

hipError_t launch_window_bwd_f16_d128(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream) {
    return launch_window_bwd<true, 128>(p, g, tile_rows, stream);
}

}  // namespace grat
