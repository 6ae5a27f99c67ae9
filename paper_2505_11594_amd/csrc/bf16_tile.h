// 16-bit tile layout in LDS of the NV16 attention kernel (the 16-bit kernels share
// the K tile's swizzle): a K tile [BKV rows][D] and a V^T tile [D rows][BKV],
// each row cut into 16-byte chunks that are XOR-swizzled against LDS bank conflicts.
#pragma once
#include "sage_common.h"

namespace sage {

template <int D, int BKV>
struct Bf16TileT {
  static constexpr int KROW = D * 2;          // bytes per K row
  static constexpr int KCH = KROW / 16;       // chunks per K row (16 or 8)
  static constexpr int VROW = BKV * 2;        // bytes per V^T tile row
  static constexpr int VCH = VROW / 16;       // chunks per V^T tile row (8 or 16)
  static constexpr int K_OFF = 0;
  static constexpr int V_OFF = BKV * KROW;
  static constexpr int BYTES = V_OFF + D * VROW;
};

// 16-byte chunk swizzle: lanes of one operand read sit on consecutive rows at
// one chunk; keep 8 (32 banks) or 16 (64 banks) consecutive rows on distinct
// bank groups.  Only row bits 0..4 matter, so a 32-row block offset does not
// change the swizzle.
template <int NCH>
__device__ __forceinline__ int bswz(int row, int ch) {
  if constexpr (NCH == 16) return ch ^ (row & 15);
  else return ch ^ (((row & 31) ^ ((row & 31) >> 3)) & 7);
}

__device__ __forceinline__ v8bf as_bf(const v4i x) { return __builtin_bit_cast(v8bf, x); }

// Chunk swizzle of the V tile (16-byte chunks of a key's row): the 8 keys whose
// chunk pairs one read instruction touches fall on distinct bank groups.
template <int D>
__device__ __forceinline__ int vswz(int row, int ch) {
  return D == 128 ? ch ^ ((row & 7) << 1) : ch ^ (((row >> 1) & 3) << 1);
}

// The A operands (V^T) of one K-step for two channel blocks: per block two
// transposing reads, at LDS byte addresses a + OFF and a + OFF8 (8 keys further on
// for 32 x 32 x 16, 16 for 16 x 16 x 32).  One asm block with its own wait: for the builtin the compiler first
// waits for every direct-to-LDS load in flight (see sage_common.h).
template <int OFF, int OFF8>
__device__ __forceinline__ void vt_read2(uint32_t a0, uint32_t a1, v8bf& r0, v8bf& r1) {
  v2u x0, x1, x2, x3;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
      "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x0), "=&v"(x1), "=&v"(x2), "=&v"(x3)
      : "v"(a0), "v"(a1), "n"(OFF), "n"(OFF8)
      : "memory");
  r0 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x0, x1, 0, 1, 2, 3));
  r1 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x2, x3, 0, 1, 2, 3));
}
// The same for four channel blocks, with one wait.
template <int OFF, int OFF8>
__device__ __forceinline__ void vt_read4(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, v8bf& r0, v8bf& r1, v8bf& r2,
                                         v8bf& r3) {
  v2u x0, x1, x2, x3, x4, x5, x6, x7;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
      "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
      "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x0), "=&v"(x1), "=&v"(x2), "=&v"(x3), "=&v"(x4), "=&v"(x5), "=&v"(x6), "=&v"(x7)
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF), "n"(OFF8)
      : "memory");
  r0 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x0, x1, 0, 1, 2, 3));
  r1 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x2, x3, 0, 1, 2, 3));
  r2 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x4, x5, 0, 1, 2, 3));
  r3 = __builtin_bit_cast(v8bf, __builtin_shufflevector(x6, x7, 0, 1, 2, 3));
}

}  // namespace sage
