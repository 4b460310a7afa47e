// Attention within a window: half, head_dim 64.
#include "sequence_fwd.h"

namespace grat {

hipError_t launch_window_fwd_f16_d64(const SelParams& p, int tile_rows, hipStream_t stream) { return launch_window<true, 64>(p, tile_rows, stream); }

}  // namespace grat
