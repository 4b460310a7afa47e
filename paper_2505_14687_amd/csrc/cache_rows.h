// Rows of a cache, written and read back (cache_rows.hip).
#pragma once
#include "sequence_common.h"

namespace grat {

struct AppendParams {
    RotaryParams p;              // Q, K, V; out: Q, K_cache, V_cache.  rot 0: nothing is turned
    SeqTensor k_scale, v_scale;  // float; 8 bits
};
hipError_t launch_cache_append(const AppendParams& a, grat_dtype dtype, bool eight, hipStream_t stream);

struct ReadParams {
    SeqTensor cache, scale, out;
    const int32_t* k_len;
    int64_t pieces;              // of 16 numbers
    FastDiv fd_items, fd_rows, fd_heads;
};
hipError_t launch_cache_read(const ReadParams& p, grat_dtype dtype, hipStream_t stream);

}  // namespace grat
