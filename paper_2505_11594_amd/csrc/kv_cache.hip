// The paged cache of keys and values: storing new tokens, and shortening cached
// sequences to their most attended tokens.  Both move rows; the bytes they read and write
// bound them, but for the 8-bit append, whose arithmetic does (below).
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
// sides are contiguous for one head.  4 sequences of up to 4096 tokens, 8 heads: 16-bit
// 15-16 us, 5.8 TB/s; INT8 19-20 us, 3.5 TB/s, as the VALU is busy 95% of the time (65%
// for 16 bits: the divisions that find a row's place).
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
// The weight of the last token that is kept comes from a radix selection from the
// top (digits of 11, 11 and 10 bits, so that the first one spreads weights of like
// size over 4 bins per power of two); then the kept indices and weights are written, and
// move copies the rows to their new pages.
//
// One workgroup per (sequence, head) does the selection in one launch where that
// fills half the GPU, or the sequences are short.  A single workgroup takes 74 us for
// 65536 tokens (its LDS atomics and scattered stores bound it), so a few long
// sequences are cut into chunks: a launch per digit leaves each chunk's histogram in
// the workspace, from which the next adds up all chunks' to pick the digit, and those in
// front of its own to find its place behind them (4 launches, 36 us).
// ---------------------------------------------------------------------------
constexpr int EV = 1024;                                 // threads of the selection
constexpr int ER = 8;                                    // neighbouring tokens per thread and round of the writing
constexpr int EL = 16;                                   // loads per thread in flight
constexpr int BINS = 2048;
constexpr int EVICT_CHUNK = EV * ER, EVICT_MOST = 16;    // tokens per chunk at least, chunks at most
static_assert(EV * 2 == BINS && EV * ER < 1 << 14, "bins per thread; counts of a round");

// Ascending in the weight as an unsigned number; -0 and 0 are equal, NaN is lowest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit_mask(int pass) { return pass == 2 ? 1023u : BINS - 1u; }

struct EvictLds {
  int hist[BINS];
  int red[EV / 64];
  int pick[2];
};

// Exclusive sum over the workgroup, and the total.
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

// What is known of the last kept key: its top digits, and how many of the tokens that
// have them are kept.
struct Last {
  uint32_t prefix, mask;
  int need;
};

// Histogram of one digit of the tokens [lo, hi) whose upper digits are known.
__device__ __forceinline__ void histogram(EvictLds& l, const float* w, int lo, int hi, int pass, const Last& last) {
  const int tid = threadIdx.x, shift = digit_shift(pass);
  const uint32_t bins = digit_mask(pass);
  for (int i = tid; i < BINS; i += EV) l.hist[i] = 0;
  __syncthreads();
  for (int j0 = lo + tid; j0 < hi; j0 += EV * EL) {
    float x[EL];
#pragma unroll
    for (int e = 0; e < EL; ++e) x[e] = w[imin(j0 + e * EV, hi - 1)];
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      const uint32_t k = weight_key(x[e]);
      if (j0 + e * EV < hi && (k & last.mask) == last.prefix) atomicAdd(&l.hist[(k >> shift) & bins], 1);
    }
  }
  __syncthreads();
}
// Thread t holds the counts c0, c1 of bins 2047 - 2 t and 2046 - 2 t: the digit of the
// need-th largest.
__device__ __forceinline__ void pick_digit(EvictLds& l, int c0, int c1, int pass, Last& last) {
  const int d = BINS - 1 - 2 * threadIdx.x;
  int total;
  const int above = block_scan(c0 + c1, l.red, &total);
  if (above < last.need && above + c0 >= last.need) {
    l.pick[0] = d;
    l.pick[1] = above;
  } else if (above + c0 < last.need && above + c0 + c1 >= last.need) {
    l.pick[0] = d - 1;
    l.pick[1] = above + c0;
  }
  __syncthreads();
  last.prefix |= (uint32_t)l.pick[0] << digit_shift(pass);
  last.mask |= digit_mask(pass) << digit_shift(pass);
  last.need -= l.pick[1];
  __syncthreads();
}

// The kept tokens of [j0, j1): those outside [lo, hi), above last.prefix, and the first
// last.need with it; `out` tokens are kept in front of j0 without the last kind, and
// `ties` of that kind lie there.
__device__ __forceinline__ void write_kept(EvictLds& l, const float* w, int32_t* kept, float* nw, int j0, int j1, int lo, int hi,
                                           bool any, const Last& last, int out, int ties) {
  for (; j0 < j1; j0 += EV * ER) {
    const int j = j0 + threadIdx.x * ER;
    float x[ER];
    uint32_t keep = 0, tie = 0;                          // bit e: token j + e
#pragma unroll
    for (int e = 0; e < ER; ++e) x[e] = j + e < j1 ? w[j + e] : 0.0f;
#pragma unroll
    for (int e = 0; e < ER; ++e) {
      const uint32_t k = weight_key(x[e]);
      const bool fixed = j + e < lo || j + e >= hi;
      if (j + e < j1 && (fixed || (any && k > last.prefix))) keep |= 1u << e;
      if (!fixed && any && k == last.prefix && j + e < j1) tie |= 1u << e;
    }
    int total;
    const int scan = block_scan(__builtin_popcount(keep) | __builtin_popcount(tie) << 16, l.red, &total);   // both below 2^14
    int kb = out + (scan & 0xFFFF), tb = ties + (scan >> 16);
    out += total & 0xFFFF;
    ties += total >> 16;
#pragma unroll
    for (int e = 0; e < ER; ++e) {
      const bool t = tie >> e & 1u;
      if ((keep >> e & 1u) || (t && tb < last.need)) {
        const int at = kb + imin(tb, last.need);
        kept[at] = j + e;
        nw[at] = x[e];
      }
      kb += keep >> e & 1u;
      tb += t;
    }
  }
}

struct EvictHead {                                       // one sequence and head
  int n, lo, hi, need;
  const float* w;
  float* nw;
  int32_t* kept;
};
__device__ __forceinline__ EvictHead evict_head(const Evict& a, int s, int h) {
  EvictHead e;
  const size_t sh = (size_t)s * a.c.Hkv + h;
  e.n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size);
  e.lo = a.keep_first;
  e.hi = e.n - a.keep_last;
  e.need = a.budget - a.keep_first - a.keep_last;        // below hi - lo if n is above the budget
  e.w = a.weights + sh * a.wstride;
  e.nw = a.new_weights + sh * a.new_wstride;
  e.kept = a.kept + sh * a.budget;
  return e;
}
// What lies behind the kept tokens, and sequences that are kept whole (then true);
// part `c` of `parts`.
__device__ __forceinline__ bool evict_ends(const Evict& a, const EvictHead& e, int s, int h, int c, int parts) {
  const int m = imin(e.n, a.budget), first = c * EV + threadIdx.x, step = parts * EV;
  if (first == 0 && h == 0) a.new_lens[s] = m;
  for (int j = m + first; j < a.budget; j += step) e.kept[j] = -1;
  const int new_capacity = a.new_max_pages * a.c.page_size;
  for (int j = m + first; j < new_capacity; j += step) e.nw[j] = 0.0f;
  if (e.n > a.budget) return false;
  for (int j = first; j < e.n; j += step) { e.kept[j] = j; e.nw[j] = e.w[j]; }
  return true;
}

__global__ __launch_bounds__(EV) void evict_select_kernel(const Evict a) {
  __shared__ EvictLds l;
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const EvictHead e = evict_head(a, s, h);
  if (evict_ends(a, e, s, h, 0, 1)) return;
  Last last = {0u, 0u, e.need};
  if (e.need > 0)
    for (int pass = 0; pass < 3; ++pass) {
      histogram(l, e.w, e.lo, e.hi, pass, last);
      pick_digit(l, l.hist[BINS - 1 - 2 * tid], l.hist[BINS - 2 - 2 * tid], pass, last);
    }
  write_kept(l, e.w, e.kept, e.nw, 0, e.n, e.lo, e.hi, e.need > 0, last, 0, 0);
}

// The same in chunks: a launch for each digit (pass 0, 1, 2), and one that writes (3).
__global__ __launch_bounds__(EV) void evict_chunk_kernel(const Evict a, int pass) {
  __shared__ EvictLds l;
  const int c = blockIdx.x, h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
  const EvictHead e = evict_head(a, s, h);
  if (pass == 3 && evict_ends(a, e, s, h, c, a.chunks)) return;
  if (e.n <= a.budget) return;
  const int b0 = imin(e.n, c * a.chunk), b1 = imin(e.n, b0 + a.chunk);
  const size_t head = (size_t)s * a.c.Hkv + h;
  int* const mine = a.hist + head * a.chunks * 3 * BINS;   // [chunk][digit][bin]
  int* const state = a.hist + (size_t)a.c.S * a.c.Hkv * a.chunks * 3 * BINS + (head * a.chunks + c) * 4;   // this chunk's, from pass to pass
  Last last = {0u, 0u, e.need};
  int out = 0, ties = 0;
  if (e.need > 0 && pass > 0) {
    const int p = pass - 1;
    if (pass > 1) {
      last.prefix = (uint32_t)state[0];
      last.need = state[1];
      out = state[2];
      for (int i = 0; i < p; ++i) last.mask |= digit_mask(i) << digit_shift(i);
    }
    // the digit before over all chunks, and over those in front of this one (bins BINS - 1 - 2 tid and the next)
    int t0 = 0, t1 = 0, f0 = 0, f1 = 0;
    const int* x = mine + p * BINS + BINS - 2 - 2 * tid;
#pragma unroll 8
    for (int k = 0; k < a.chunks; ++k) {
      const v2u y = *reinterpret_cast<const v2u*>(x + (size_t)k * 3 * BINS);
      t0 += (int)y[1]; t1 += (int)y[0];
      if (k < c) { f0 += (int)y[1]; f1 += (int)y[0]; }
    }
    const int d = BINS - 1 - 2 * tid;
    pick_digit(l, t0, t1, p, last);
    const int at = (int)(last.prefix >> digit_shift(p) & digit_mask(p));
    int total;
    block_scan((d > at ? f0 : 0) + (d - 1 > at ? f1 : 0), l.red, &total);
    out += total;
    if (pass == 3) {
      block_scan((d == at ? f0 : 0) + (d - 1 == at ? f1 : 0), l.red, &ties);
    } else if (tid == 0) {                               // (all have read it: the scans' barriers)
      state[0] = (int)last.prefix;
      state[1] = last.need;
      state[2] = out;
    }
  }
  if (pass == 3) {
    out += imin(b0, e.lo) + imax(0, b0 - e.hi);          // first and last tokens before the chunk
    write_kept(l, e.w, e.kept, e.nw, b0, b1, e.lo, e.hi, e.need > 0, last, out, ties);
  } else if (e.need > 0) {
    histogram(l, e.w, imax(e.lo, b0), imin(e.hi, b1), pass, last);
    int* x = mine + ((size_t)c * 3 + pass) * BINS;
    for (int i = tid; i < BINS; i += EV) x[i] = l.hist[i];
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

int evict_chunks(int S, int Hkv, int capacity) {
  if ((long long)S * Hkv >= 128 || capacity <= 2 * EVICT_CHUNK) return 1;
  return imin(EVICT_MOST, cdiv(capacity, EVICT_CHUNK));
}
size_t evict_hist_ints(int S, int Hkv, int capacity) {
  const int c = evict_chunks(S, Hkv, capacity);
  return c > 1 ? (size_t)S * Hkv * c * (3 * BINS + 4) : 0;
}

hipError_t launch_kv_evict(const Evict& x, int D, hipStream_t st) {
  Evict a = x;
  const int capacity = a.c.max_pages * a.c.page_size;
  a.chunks = evict_chunks(a.c.S, a.c.Hkv, capacity);
  a.chunk = cdiv(cdiv(capacity, a.chunks), EVICT_CHUNK) * EVICT_CHUNK;
  hipError_t e = hipSuccess;
  if (a.chunks > 1) {
    for (int pass = 0; pass < 4 && e == hipSuccess; ++pass) {
      hipLaunchKernelGGL(evict_chunk_kernel, dim3((unsigned)a.chunks, (unsigned)a.c.Hkv, (unsigned)a.c.S), dim3(EV), 0, st, a, pass);
      e = hipGetLastError();
    }
  } else {
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)a.c.S, (unsigned)a.c.Hkv), dim3(EV), 0, st, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  const int elem = a.c.k_scale ? 1 : 2, rb = D * elem, per = 256 / (rb / 16);
  const dim3 grid((unsigned)imin(cdiv(a.budget, per), imax(1, (int)(8192 / ((long long)a.c.S * a.c.Hkv)))),
                  (unsigned)a.c.Hkv, (unsigned)a.c.S);
  if (rb == 256) hipLaunchKernelGGL((evict_move_kernel<256>), grid, dim3(256), 0, st, a, elem);
  else if (rb == 128) hipLaunchKernelGGL((evict_move_kernel<128>), grid, dim3(256), 0, st, a, elem);
  else hipLaunchKernelGGL((evict_move_kernel<64>), grid, dim3(256), 0, st, a, elem);
  return hipGetLastError();
}

}  // namespace sage
