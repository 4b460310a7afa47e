// What the host sides of the token-sequence operators check alike.
#pragma once
#include "sequence_common.h"

namespace grat {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool is16(grat_dtype t) { return t == GRAT_BF16 || t == GRAT_F16; }
inline bool known(grat_dtype t) { return is16(t) || t == GRAT_F32; }

// A tensor whose rows are read or written as 16-byte vectors.
inline grat_status check_tensor(const grat_tensor* t, grat_dtype dtype, int32_t head_dim) {
    if (!t || !t->data) return GRAT_ERR_NULL;
    if (t->stride_n < head_dim || t->stride_b < 0 || t->stride_h < 0) return GRAT_ERR_BAD_DIMS;
    const int vec = is16(dtype) ? 8 : 4;
    if (t->stride_n % vec || t->stride_b % vec || t->stride_h % vec || !aligned16(t->data)) return GRAT_ERR_UNSUPPORTED;
    if (t->stride_n >= ((int64_t)1 << 24) || t->stride_b >= ((int64_t)1 << 46) || t->stride_h >= ((int64_t)1 << 46))
        return GRAT_ERR_UNSUPPORTED;
    return GRAT_OK;
}

// ... and one that is written to: its rows may not lie on each other.
inline grat_status check_output(const grat_tensor* t, grat_dtype dtype, int32_t head_dim, int32_t batch, int32_t heads) {
    const grat_status st = check_tensor(t, dtype, head_dim);
    return st == GRAT_OK && ((batch > 1 && t->stride_b == 0) || (heads > 1 && t->stride_h == 0)) ? GRAT_ERR_BAD_DIMS : st;
}

inline SeqTensor of(const grat_tensor* t) { return {(uint8_t*)t->data, t->stride_b, t->stride_h, t->stride_n}; }

constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // of an axis of a launch; fewer

inline grat_status status_of(hipError_t e) { return e == hipSuccess ? GRAT_OK : GRAT_ERR_HIP; }

grat_status make_rotary(const grat_rotary_args* a, bool with_k, RotaryParams* out);   // (sequence_api.hip)

// Shares of the caller's scratch memory, counted from its start (which is null where only the bytes are asked for).
struct Scratch {
    uint8_t* base;
    int64_t bytes = 0;
    template <typename T>
    T* take(int64_t n) {
        T* const at = (T*)(base + bytes);
        bytes += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
        return at;
    }
};

}  // namespace grat
