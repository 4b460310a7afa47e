// A slice of the gradient kernels' instantiations (sequence_bwd.h).
#include "sequence_bwd.h"

namespace grat {
hipError_t launch_selected_bwd_f16_d128(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream) {
    return launch_bwd<true, 128>(p, g, tile_rows, tile_keys, stream);
}
}  // namespace grat
