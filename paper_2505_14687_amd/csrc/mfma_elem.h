// What the 16-bit attention kernels share: fragments of the matrix instruction, what depends on the element type, and the
// exchange between the two halves of a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace grat {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) short frag8;   // 8 sixteen-bit elements of either type
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

#define LDS_PTR(T) __attribute__((address_space(3))) T*

// What depends on the 16-bit element type (F16 = false: bfloat16, true: IEEE half).  Fragments
// travel as type-neutral frag8 and are reinterpreted at the MFMA.
template <bool F16>
struct Elem {
    // a lane's block row sum (16 weights) beyond this forces a new reference maximum: every single
    // weight then stays inside the type's range (half: 65504) with its full relative precision
    static constexpr float kSumLimit = F16 ? 0x1p+15f : 0x1p+40f;
    static __device__ __forceinline__ f32x16 mfma(frag8 a, frag8 b, f32x16 c) {
        if constexpr (F16)
            return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(frag8 a, frag8 b, f32x4 c) {   // 16x16x32
        if constexpr (F16)
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    // two fp32 values rounded to nearest-even and packed (lo in the low half)
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const f32x2 v = {lo, hi};
        if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
        else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    }
};

// Exchange between the two lanes that hold the same query (lane and lane ^ 32) with one
// v_permlane32_swap.  The two results are copied to scalars before they are reinterpreted:
// a bit cast applied directly to a vector element reads element 0 with this compiler.
__device__ __forceinline__ void swap_halves(float x, float& lower, float& upper) {
    const uint32_t a = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    lower = __builtin_bit_cast(float, r0);   // value held by the lane with the same query, half 0
    upper = __builtin_bit_cast(float, r1);   // ... half 1
}
__device__ __forceinline__ float max_across_halves(float x) {
    float lo, hi;
    swap_halves(x, lo, hi);
    return fmaxf(lo, hi);
}
__device__ __forceinline__ float sum_across_halves(float x) {
    float lo, hi;
    swap_halves(x, lo, hi);
    return lo + hi;
}

}  // namespace grat
