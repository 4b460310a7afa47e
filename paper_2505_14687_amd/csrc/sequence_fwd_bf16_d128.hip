// A slice of the forward kernel's instantiations (sequence_fwd.h).
#include "sequence_fwd.h"

namespace grat {
hipError_t launch_selected_fwd_bf16_d128(const SelParams& p, int tile_rows, hipStream_t stream) {
    return launch_fwd<false, 128>(p, tile_rows, stream);
}
}  // namespace grat
