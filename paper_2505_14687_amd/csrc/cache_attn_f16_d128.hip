// Attention over a cache: half, head_dim 128.
#include "cache_attn.h"

namespace grat {

hipError_t launch_cache_attention_f16_d128(const SelParams& p, bool eight, int tile_rows, hipStream_t stream) {
    return launch_cache_attention<true, 128>(p, eight, tile_rows, stream);
}

}  // namespace grat
