// The split of one-token attention over a paged cache, which its kernels share: the
// visible tiles of DT keys of all sequences, in steps of DW tiles, form one line that
// the workgroups of a key head cut into equal shares (attn_decode.hip says more).
#pragma once
#include "lm_args.h"
#include "mma16.h"
#include "window.h"

namespace sage {

constexpr int DG = 16;                  // query heads per workgroup

__device__ __forceinline__ float max_over_groups(float x) {      // over the lanes l % 16 equal
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = smax(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return smax(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Tiles of a sequence.
template <int DT>
__device__ __forceinline__ TileList seq_tiles(const Decode& a, int s, int* n) {
  *n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size);
  return decode_tiles(*n, a.window, a.sinks, DT);
}

// The line of all sequences' steps.  Up to 64 sequences each wave adds up their steps
// itself, one per lane; of more, line_kernel has left the steps before each in
// a.before.
constexpr int LINE = 64;
// a / b (b > 0, a >= 0), in 32 bits where they do: a 64-bit division takes some 150 instructions.
__device__ __forceinline__ long long divide(long long a, long long b) {
  if ((unsigned long long)(a | b) < 1ull << 32) return (uint32_t)a / (uint32_t)b;
  return a / b;
}
struct Line {
  long long total, share;               // steps in all, and per workgroup
};
template <int DT, int DW>
__device__ __forceinline__ int steps_of_lane(const Decode& a, int* n) {      // (n: the length)
  const int lane = threadIdx.x & 63;
  *n = 0;
  return lane < a.c.S ? cdiv(seq_tiles<DT>(a, lane, n).count, DW) : 0;
}
template <int DT, int DW>
__device__ __forceinline__ int steps_of_lane(const Decode& a) {
  int n;
  return steps_of_lane<DT, DW>(a, &n);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_lanes(int x) {        // lanes that the control does not reach add 0
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int lanes_up_to(int x) {      // inclusive sum over the lanes
  x = add_lanes<0x111, 0xF>(x);                          // within rows of 16: from 1, 2, 4, 8 lanes before
  x = add_lanes<0x112, 0xF>(x);
  x = add_lanes<0x114, 0xF>(x);
  x = add_lanes<0x118, 0xF>(x);
  x = add_lanes<0x142, 0xA>(x);                          // a row's last lane to the next row, lane 31 to the upper half
  return add_lanes<0x143, 0xC>(x);
}
__device__ __forceinline__ Line steps_line(const Decode& a, int sum) {
  Line l;
  l.total = a.before ? a.before[a.c.S] : __shfl(sum, 63, 64);
  l.share = divide(l.total + a.nw - 1, a.nw);
  return l;
}
// The sequence that holds step r < total, and the steps before it (c: this lane's
// steps, sum: up to it).
__device__ __forceinline__ int find_step(const Decode& a, int c, int sum, long long r, long long* before) {
  const int lane = threadIdx.x & 63;
  if (!a.before) {
    const int first = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > r));
    *before = __shfl(sum - c, first, 64);
    return first;
  }
  // the first s with before[s + 1] > r: 64 places are looked at at a time
  int lo = 0, len = a.c.S;                               // it is in [lo, lo + len)
  while (len > 1) {
    const int step = cdiv(len, 64), s = lo + (lane + 1) * step;   // up to s: before[s] > r?
    const unsigned long long past = __builtin_amdgcn_ballot_w64(s >= lo + len || a.before[s] > r);
    const int first = __builtin_ctzll(past);
    len = imin(step, len - first * step);
    lo += first * step;
  }
  *before = a.before[lo];
  return lo;
}

// Steps before each of many sequences, and in all.  One workgroup.
template <int DT, int DW>
__global__ __launch_bounds__(1024) void line_kernel(const Decode a) {
  __shared__ int red[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long long base = 0;
  for (int s0 = 0; s0 < a.c.S; s0 += 1024) {
    int n, c = 0;
    if (s0 + tid < a.c.S) c = cdiv(seq_tiles<DT>(a, s0 + tid, &n).count, DW);
    const int sum = lanes_up_to(c);
    __syncthreads();
    if (lane == 63) red[wave] = sum;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += red[w];
      all += red[w];
    }
    if (s0 + tid < a.c.S) a.before[s0 + tid] = base + before + sum - c;
    base += all;
  }
  if (tid == 0) a.before[a.c.S] = base;
}

}  // namespace sage
