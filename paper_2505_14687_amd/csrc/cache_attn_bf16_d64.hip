// Attention over a cache: bfloat16, head_dim 64.
#include "cache_attn.h"

namespace grat {

hipError_t launch_cache_attention_bf16_d64(const SelParams& p, bool eight, int tile_rows, hipStream_t stream) {
    return launch_cache_attention<false, 64>(p, eight, tile_rows, stream);
}

}  // namespace grat
