// Attention within a window: bfloat16, head_dim 64.
#include "sequence_fwd.h"

namespace grat {

hipError_t launch_window_fwd_bf16_d64(const SelParams& p, int tile_rows, hipStream_t stream) { return launch_window<false, 64>(p, tile_rows, stream); }

}  // namespace grat
