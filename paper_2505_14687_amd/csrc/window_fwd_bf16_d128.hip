// Attention within a window: bfloat16, head_dim 128.
#include "sequence_fwd.h"

namespace grat {

hipError_t launch_window_fwd_bf16_d128(const SelParams& p, int tile_rows, hipStream_t stream) { return launch_window<false, 128>(p, tile_rows, stream); }

}  // namespace grat
