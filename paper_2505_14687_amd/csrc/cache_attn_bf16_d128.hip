// Attention over a cache: bfloat16, head_dim 128.
#include "cache_attn.h"

namespace grat {

hipError_t launch_cache_attention_bf16_d128(const SelParams& p, bool eight, int tile_rows, hipStream_t stream) {
    return launch_cache_attention<false, 128>(p, eight, tile_rows, stream);
}

}  // namespace grat
