// The 16-bit matrix instructions in the input's type, on operands held as bits, and
// their operands' places in LDS tiles.
#pragma once
#include "bf16_tile.h"

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

// Probabilities enter the second product in 16 bits.  In fp16 the one-token attention
// and the backward carry them 2^15 larger: probabilities down to 2^-29 of the row's
// maximum stay normal numbers instead of those above 2^-14 only, and the largest is
// 2^15 < 65504.  (The window forward carries 2^7, as its maximum may lag by 2^8: normal
// down to 2^-21 of that maximum.)  The sums carry the same factor and lose it in the final
// division.  bf16 has the range of fp32 and needs none.
template <bool BF16> constexpr float kPShift = BF16 ? 0.0f : 15.0f;

// A lane's LDS addresses in a tile at offset 0 of LDS: rows start on multiples of
// their size, so the swizzled chunk is or-ed in, and the other chunks follow by xor with
// constants: row_at ^ 32 i is chunk 2 i + hi of row l % 32, tr_at ^ 64 db the piece of
// channel block db of the transposing read (see attn_bf16.hip).  They are made
// opaque where they are used, as the compiler would keep every one in a register.
// (Tiles that are only read by rows are swizzled with bswz.)
template <int D, bool ROWS_ONLY = false>
__device__ __forceinline__ uint32_t row_at() {
  const int lane = threadIdx.x & 63, col = lane & 31, hi = lane >> 5;
  return col * (D * 2) + (ROWS_ONLY ? bswz<D / 8>(col, hi) : vswz<D>(col, hi)) * 16;
}
template <int D>
__device__ __forceinline__ uint32_t tr_at() {
  const int lane = threadIdx.x & 63, hi = lane >> 5;
  const int r = 4 * hi + (lane & 15) / 4, c0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  return r * (D * 2) + vswz<D>(r, c0) * 16 + 8 * (lane & 1);
}
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ v4i lds16(uint32_t at) { return *(const __attribute__((address_space(3))) v4i*)(uintptr_t)at; }
__device__ __forceinline__ v4f lds4f(uint32_t at) { return *(const __attribute__((address_space(3))) v4f*)(uintptr_t)at; }

// acc (dims x columns) += the transpose of 16 rows OFF bytes behind `at` times b.
template <int D, bool BF16, int OFF>
__device__ __forceinline__ void cols_times(uint32_t at, const v4i b, v16f* acc) {
  v8bf x[D / 32];
  if constexpr (D == 128) vt_read4<OFF, OFF + 8 * D * 2>(at, at ^ 64, at ^ 128, at ^ 192, x[0], x[1], x[2], x[3]);
  else vt_read2<OFF, OFF + 8 * D * 2>(at, at ^ 64, x[0], x[1]);
#pragma unroll
  for (int db = 0; db < D / 32; ++db) acc[db] = mma32<BF16>(__builtin_bit_cast(v4i, x[db]), b, acc[db]);
}

}  // namespace sage
