// The paged cache of keys and values: storing new tokens, and shortening cached
// sequences to their most attended tokens.  Both move rows and are bound by the
// bytes they read and write.
#include "lm_args.h"
#include "sage_common.h"
#include "window.h"

namespace sage {


constexpr float kRound = 12582912.0f;                    // 1.5 * 2^23: adding it rounds to an integer, ties to even

// 16 bytes of a row of new tokens into the cache; for an 8-bit cache 8 codes of
//   s = max|x| / 127 over the row,  code = rint(x * fl32(1 / s))
// where the D / 8 lanes of the row exchange the maximum.  Rows whose scale is below
// the smallest normal number (1 / s could overflow) have s = 0 and codes 0.
template <int D, bool BF16>
__device__ __forceinline__ void quantize8(const v4i x, float* scale, v2u* codes) {
  float v[8], amax = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = widen<BF16>((uint16_t)((uint32_t)x[i / 2] >> (16 * (i & 1))));
    amax = __builtin_fmaxf(amax, __builtin_fabsf(v[i]));
  }
#pragma unroll
  for (int o = D / 16; o >= 1; o >>= 1) amax = __builtin_fmaxf(amax, __shfl_xor(amax, o, 64));
  float s = amax / 127.0f, r = 0.0f;                     // correctly rounded divisions
  if (s >= 0x1p-126f) r = 1.0f / s;
  else s = 0.0f;
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i] * r + kRound) & 0xFFu;
  *scale = s;
  *codes = v2u{w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24};
}

// D / 8 lanes per row; rows in the order (sequence, head, token), in which both
// sides are contiguous for one head.
template <int D, bool BF16, bool I8>
__global__ __launch_bounds__(256) void kv_append_kernel(const Append a) {
  constexpr int LPR = D / 8;
  const int ch = threadIdx.x % LPR;
  const long long row = (long long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const int hn = a.c.Hkv * a.N;
  const int s = (int)(row / hn), rest = (int)(row - (long long)s * hn), h = rest / a.N, t = rest - h * a.N;
  if (s >= a.c.S) return;
  const int count = a.counts ? a.counts[s] : a.N;
  const long long at = (long long)a.pos[s] + t;
  const long long capacity = (long long)a.c.max_pages * a.c.page_size;
  bool ok = t < count && at >= 0 && at < capacity;
  int page = 0, slot = 0;
  if (ok) {
    page = a.c.table[(size_t)s * a.c.max_pages + (int)at / a.c.page_size];
    slot = (int)at % a.c.page_size;
    ok = page_ok(page, a.c.pages);
  }
  if (!ok) return;                                       // a row's lanes leave together
  const uint16_t* k = (const uint16_t*)a.k + (s * a.ks.b + h * a.ks.h + t * a.ks.n) + 8 * ch;
  const uint16_t* v = (const uint16_t*)a.v + (s * a.vs.b + h * a.vs.h + t * a.vs.n) + 8 * ch;
  const v4i kx = *reinterpret_cast<const v4i*>(k), vx = *reinterpret_cast<const v4i*>(v);
  const long long kd = page * a.c.ks.b + h * a.c.ks.h + slot * a.c.ks.n + 8 * ch;
  const long long vd = page * a.c.vs.b + h * a.c.vs.h + slot * a.c.vs.n + 8 * ch;
  if constexpr (I8) {
    const size_t sc = ((size_t)page * a.c.Hkv + h) * a.c.page_size + slot;
    float x;
    v2u c;
    quantize8<D, BF16>(kx, &x, &c);
    *reinterpret_cast<v2u*>((uint8_t*)a.c.k + kd) = c;
    if (ch == 0) const_cast<float*>(a.c.k_scale)[sc] = x;
    quantize8<D, BF16>(vx, &x, &c);
    *reinterpret_cast<v2u*>((uint8_t*)a.c.v + vd) = c;
    if (ch == 0) const_cast<float*>(a.c.v_scale)[sc] = x;
  } else {
    *reinterpret_cast<v4i*>((uint16_t*)a.c.k + kd) = kx;
    *reinterpret_cast<v4i*>((uint16_t*)a.c.v + vd) = vx;
  }
  if (a.weights && ch == 0) a.weights[((size_t)s * a.c.Hkv + h) * a.wstride + at] = 0.0f;
}

hipError_t launch_kv_append(const Append& a, int D, bool bf16, hipStream_t st) {
  const long long rows = (long long)a.c.S * a.c.Hkv * a.N;
  const int per = 256 / (D / 8);
  const dim3 grid((unsigned)((rows + per - 1) / per)), block(256);
  const bool i8 = a.c.k_scale != nullptr;
#define SAGE_APPEND(DD, BB)                                                                      \
  if (i8) hipLaunchKernelGGL((kv_append_kernel<DD, BB, true>), grid, block, 0, st, a);           \
  else hipLaunchKernelGGL((kv_append_kernel<DD, BB, false>), grid, block, 0, st, a);             \
  return hipGetLastError()
  if (D == 128) {
    if (bf16) { SAGE_APPEND(128, true); }
    SAGE_APPEND(128, false);
  }
  if (bf16) { SAGE_APPEND(64, true); }
  SAGE_APPEND(64, false);
#undef SAGE_APPEND
}

// ---------------------------------------------------------------------------
// Eviction.  A sequence of n > budget cached tokens keeps, per key head, its first
// keep_first and last keep_last tokens and the heaviest of those between, ties
// with the lowest index first, in ascending order.
//
// select: one workgroup per (sequence, head) finds the weight of the last token
// that is kept (a radix selection: 4 passes over 8-bit digits, from the top) and
// writes the kept indices and weights.  move: the kept rows to their new pages.
// ---------------------------------------------------------------------------
constexpr int EV = 1024;                                 // threads of the selection

// Ascending in the weight as an unsigned number; -0 and 0 are equal, NaN is lowest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sum over the workgroup, and the total.  `red`: 16 words of LDS.
__device__ __forceinline__ int block_scan(int x, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(inc, o, 64);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 63) red[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < EV / 64; ++w) {
    if (w < wave) before += red[w];
    all += red[w];
  }
  *total = all;
  return before + inc - x;
}

__global__ __launch_bounds__(EV) void evict_select_kernel(const Evict a) {
  __shared__ int hist[256];
  __shared__ int red[EV / 64];
  __shared__ int pick[2];
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const int n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size);
  const size_t sh = (size_t)s * a.c.Hkv + h;
  const float* w = a.weights + sh * a.wstride;
  float* nw = a.new_weights + sh * a.new_wstride;
  int32_t* kept = a.kept + sh * a.budget;
  const int m = imin(n, a.budget);
  if (tid == 0 && h == 0) a.new_lens[s] = m;
  for (int j = m + tid; j < a.budget; j += EV) kept[j] = -1;
  const int new_capacity = a.new_max_pages * a.c.page_size;
  for (int j = m + tid; j < new_capacity; j += EV) nw[j] = 0.0f;
  if (n <= a.budget) {
    for (int j = tid; j < n; j += EV) { kept[j] = j; nw[j] = w[j]; }
    return;
  }
  const int lo = a.keep_first, hi = n - a.keep_last;     // the tokens between are chosen from
  int need = a.budget - a.keep_first - a.keep_last;      // < hi - lo
  uint32_t prefix = 0, mask = 0;                         // digits found so far
  if (need > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += EV) hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += EV) {
        const uint32_t k = weight_key(w[j]);
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1);
      }
      __syncthreads();
      // the digit of the need-th largest: thread t holds digit 255 - t
      const int c = tid < 256 ? hist[255 - tid] : 0;
      int total;
      const int above = block_scan(c, red, &total);
      if (tid < 256 && above < need && above + c >= need) {
        pick[0] = 255 - tid;
        pick[1] = above;
      }
      __syncthreads();
      prefix |= (uint32_t)pick[0] << shift;
      mask |= 255u << shift;
      need -= pick[1];
      __syncthreads();
    }
  // `prefix` is the last kept key, `need` of the tokens that have it are kept
  const bool any = a.budget - a.keep_first - a.keep_last > 0;
  int out = 0, ties = 0;
  for (int j0 = 0; j0 < n; j0 += EV) {
    const int j = j0 + tid;
    bool keep = false, tie = false;
    if (j < n) {
      if (j < lo || j >= hi) keep = true;
      else if (any) {
        const uint32_t k = weight_key(w[j]);
        keep = k > prefix;
        tie = k == prefix;
      }
    }
    int total;
    const int tb = ties + block_scan(tie, red, &total);
    ties += total;
    if (tie && tb < need) keep = true;
    const int at = out + block_scan(keep, red, &total);
    out += total;
    if (keep) {
      kept[at] = j;
      nw[at] = w[j];
    }
  }
}

// 16 bytes per thread.  A row whose new place is its old one is left alone.
template <int RB>                                        // bytes of a row
__global__ __launch_bounds__(256) void evict_move_kernel(const Evict a, int elem) {
  constexpr int LPR = RB / 16;
  const int s = blockIdx.z, h = blockIdx.y, ch = threadIdx.x % LPR;
  const int n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size), m = imin(n, a.budget);
  const int32_t* kept = a.kept + ((size_t)s * a.c.Hkv + h) * a.budget;
  const int ps = a.c.page_size;
  for (int j = blockIdx.x * (256 / LPR) + threadIdx.x / LPR; j < m; j += gridDim.x * (256 / LPR)) {
    const int src = kept[j];
    const int sp = a.c.table[(size_t)s * a.c.max_pages + src / ps], ss = src % ps;
    const int dp = a.new_table[(size_t)s * a.new_max_pages + j / ps], ds = j % ps;
    if (!page_ok(sp, a.c.pages) || !page_ok(dp, a.c.pages) || (sp == dp && ss == ds)) continue;
    const uint8_t *k = (const uint8_t*)a.c.k, *v = (const uint8_t*)a.c.v;
    const v4i kx = *reinterpret_cast<const v4i*>(k + elem * (sp * a.c.ks.b + h * a.c.ks.h + ss * a.c.ks.n) + 16 * ch);
    const v4i vx = *reinterpret_cast<const v4i*>(v + elem * (sp * a.c.vs.b + h * a.c.vs.h + ss * a.c.vs.n) + 16 * ch);
    *reinterpret_cast<v4i*>(const_cast<uint8_t*>(k) + elem * (dp * a.c.ks.b + h * a.c.ks.h + ds * a.c.ks.n) + 16 * ch) = kx;
    *reinterpret_cast<v4i*>(const_cast<uint8_t*>(v) + elem * (dp * a.c.vs.b + h * a.c.vs.h + ds * a.c.vs.n) + 16 * ch) = vx;
    if (a.c.k_scale && ch == 0) {
      const size_t si = ((size_t)sp * a.c.Hkv + h) * ps + ss, di = ((size_t)dp * a.c.Hkv + h) * ps + ds;
      const_cast<float*>(a.c.k_scale)[di] = a.c.k_scale[si];
      const_cast<float*>(a.c.v_scale)[di] = a.c.v_scale[si];
    }
  }
}

hipError_t launch_kv_evict(const Evict& a, int D, hipStream_t st) {
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)a.c.S, (unsigned)a.c.Hkv), dim3(EV), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int elem = a.c.k_scale ? 1 : 2, rb = D * elem, per = 256 / (rb / 16);
  const dim3 grid((unsigned)imin(cdiv(a.budget, per), imax(1, 8192 / imax(1, imin(8192, a.c.S * a.c.Hkv)))),
                  (unsigned)a.c.Hkv, (unsigned)a.c.S);
  if (rb == 256) hipLaunchKernelGGL((evict_move_kernel<256>), grid, dim3(256), 0, st, a, elem);
  else if (rb == 128) hipLaunchKernelGGL((evict_move_kernel<128>), grid, dim3(256), 0, st, a, elem);
  else hipLaunchKernelGGL((evict_move_kernel<64>), grid, dim3(256), 0, st, a, elem);
  return hipGetLastError();
}

}  // namespace sage
