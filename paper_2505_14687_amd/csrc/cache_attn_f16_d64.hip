// Attention over a cache: half, head_dim 64.
#include "cache_attn.h"

namespace grat {

hipError_t launch_cache_attention_f16_d64(const SelParams& p, bool eight, int tile_rows, hipStream_t stream) {
    return launch_cache_attention<true, 64>(p, eight, tile_rows, stream);
}

}  // namespace grat
