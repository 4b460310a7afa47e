// Attention over a cache: bfloat16, head_dim 64.
#include "cache_attn.h"

namespace grat {

hipError_t launch_cache_attention_bf16_d64(const CacheParams& c, bool eight, int sets, hipStream_t stream) {
    return launch_cache_attention<false, 64>(c, eight, sets, stream);
}

}  // namespace grat
