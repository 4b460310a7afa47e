// Attention within a window: half, head_dim 128.
#include "sequence_fwd.h"

namespace grat {

hipError_t launch_window_fwd_f16_d128(const SelParams& p, int tile_rows, hipStream_t stream) { return launch_window<true, 128>(p, tile_rows, stream); }

}  // namespace grat
