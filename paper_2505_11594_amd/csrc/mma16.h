// The 16-bit matrix instructions in the input's type, on operands held as bits.
#pragma once
#include "sage_common.h"

namespace sage {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

template <bool BF16>
__device__ __forceinline__ v16f mma32(const v4i a, const v4i b, const v16f c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ v4f mma16(const v4i a, const v4i b, const v4f c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// Two fp32 values rounded to nearest even into one register, a in the low half.
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b});
  else return __builtin_bit_cast(uint32_t, v2h{(_Float16)a, (_Float16)b});
}

// c + the sum of a register's two 16-bit values.
template <bool BF16>
__device__ __forceinline__ float add_pair(uint32_t x, float c) {
  if constexpr (BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, x), __builtin_bit_cast(v2bf, 0x3F803F80u), c, false);
  else return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, x), __builtin_bit_cast(v2h, 0x3C003C00u), c, false);
}

// Probabilities enter the second product in 16 bits.  In fp16 they are carried
// 2^15 larger: probabilities down to 2^-29 of the row's maximum stay normal
// numbers instead of those above 2^-14 only, and the largest is 2^15 < 65504.  The
// sums carry the same factor and lose it in the final division.  bf16 has the
// range of fp32 and needs none.
template <bool BF16> constexpr float kPShift = BF16 ? 0.0f : 15.0f;

}  // namespace sage
