// The paged cache of keys and values: storing new tokens by tables or by slots, and shortening cached
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
// kv_store_kernel below, whose divisions are multiplications, in its place (graphs of calls on four sets of
// inputs, bf16, 8 heads, D = 128, pages of 32): 4 x up to 4096 tokens 16-bit 20.8 us for 20.7 here, INT8 16.3
// for 18.3; 8 x up to 1500 13.9 for 13.7, 11.4 for 12.4; 32 x 512 28.5 for 28.3, 23.9 for 24.6; 128 x 1
// 2.4 for 2.6, 3.0 for 3.1.  16-bit caches gain nothing; INT8 ones would gain 3 to 11% and are still
// stored here.
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

// The same for a cache in MXFP4, and for every kind of cache where the caller gives each
// token's slot (page * page_size + its place in the page) in place of tables (the tokens above by slots,
// in one row: 16-bit 20.1, 12.2, 27.9, 2.3 us; INT8 15.6, 10.8, 23.8, 2.9; MXFP4 11.1, 8.7, 19.0, 2.6).  MXFP4 rows:
// per 32 channels the scale 2^e has the smallest e with 6 * 2^e >= max|x| (phi of the FP4
// attention), codes are E2M1 of x / 2^e, nearest, ties to even; 4 lanes of 8 channels make
// a block.  (4 sequences of up to 4096 tokens, 8 heads: 13.3 us, 4.3 TB/s, VALU busy 43%; 14.2 with
// values widened before their conversion, divisions per row and loads behind the look-up.)
typedef uint16_t v2us __attribute__((ext_vector_type(2)));
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}
// 8 values of a block whose 32 are in 4 lanes.  Sizes of 16-bit values are in the order of their
// bits; the conversion takes pairs of them and the scale's exponent (not that of a scale below
// 2^-126, which 8 values are multiplied by).
template <bool BF16>
__device__ __forceinline__ uint32_t quantize_fp4(const v4i x, int* scale) {
  v2us big = __builtin_bit_cast(v2us, x[0] & 0x7FFF7FFF);
#pragma unroll
  for (int i = 1; i < 4; ++i) big = __builtin_elementwise_max(big, __builtin_bit_cast(v2us, x[i] & 0x7FFF7FFF));
  const uint32_t top = max_dpp<0x4E>(max_dpp<0xB1>(max((uint32_t)big[0], (uint32_t)big[1])));     // lanes ^ 1, ^ 2
  const int e = e8m0_exponent(widen<BF16>((uint16_t)top));
  *scale = e + 127;
  uint32_t c = 0;
  if (BF16 && e == -127) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = widen<BF16>((uint16_t)((uint32_t)x[i / 2] >> (16 * (i & 1)))) * 0x1p127f;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], 1.0f, 3);
  }
  const float f = __uint_as_float((uint32_t)imax(e + 127, 1) << 23);      // (fp16: -127 is a block of zeros)
  const int x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];  // (a bit cast of a vector's element would take the first one's)
  if constexpr (BF16) {
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2b, x0), f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2b, x1), f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2b, x2), f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2b, x3), f, 3);
  } else {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2h, x0), f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2h, x1), f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2h, x2), f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2h, x3), f, 3);
  }
}

struct Store {
  Append a;
  const int64_t* slots;
  Divide heads_tokens, tokens, page;
};
// TILED: a workgroup's rows are tokens of one sequence and head.
template <int D, bool BF16, int KIND, bool SLOTS, bool TILED>
__global__ __launch_bounds__(256) void kv_store_kernel(const Store st) {
  const Append& a = st.a;
  constexpr int LPR = D / 8;
  const int ch = threadIdx.x % LPR;
  int s, h, t;
  if constexpr (TILED) {
    s = blockIdx.z;
    h = blockIdx.y;
    t = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (t >= a.N) return;
  } else {
    const int row = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;        // (fewer than 2^28 rows)
    s = st.heads_tokens(row);
    const int rest = row - s * st.heads_tokens.by;
    h = st.tokens(rest);
    t = rest - h * a.N;
    if (s >= a.c.S) return;
  }
  long long page = 0, at = 0, where = 0;
  if constexpr (SLOTS) {
    where = st.slots[(long long)s * a.N + t];
  } else {
    const int count = a.counts ? a.counts[s] : a.N;
    at = (long long)a.pos[s] + t;
    if (t >= count || at < 0 || at >= (long long)a.c.max_pages * a.c.page_size) return;
    page = a.c.table[(size_t)s * a.c.max_pages + st.page((int)at)];
  }
  // (the rows are on their way while their place is looked up)
  const uint16_t* k = (const uint16_t*)a.k + (s * a.ks.b + h * a.ks.h + t * a.ks.n) + 8 * ch;
  const uint16_t* v = (const uint16_t*)a.v + (s * a.vs.b + h * a.vs.h + t * a.vs.n) + 8 * ch;
  const v4i kx = *reinterpret_cast<const v4i*>(k), vx = *reinterpret_cast<const v4i*>(v);
  int slot;
  if constexpr (SLOTS) {
    if (where < 0) return;                               // a row's lanes leave together
    page = where < (1ll << 31) ? (long long)st.page((int)where) : where / st.page.by;
    slot = (int)(where - page * st.page.by);
  } else {
    slot = (int)at - st.page((int)at) * st.page.by;
  }
  if (page < 0 || page >= a.c.pages) return;
  const long long kd = page * a.c.ks.b + h * a.c.ks.h + slot * a.c.ks.n;
  const long long vd = page * a.c.vs.b + h * a.c.vs.h + slot * a.c.vs.n;
  const size_t sc = ((size_t)page * a.c.Hkv + h) * st.page.by + slot;
  if constexpr (KIND == kCacheFp4) {
    int ke, ve;
    const uint32_t kc = quantize_fp4<BF16>(kx, &ke), vc = quantize_fp4<BF16>(vx, &ve);
    *reinterpret_cast<uint32_t*>((uint8_t*)a.c.k + kd + 4 * ch) = kc;
    *reinterpret_cast<uint32_t*>((uint8_t*)a.c.v + vd + 4 * ch) = vc;
    if ((ch & 3) == 0) {
      ((uint8_t*)const_cast<float*>(a.c.k_scale))[sc * (D / 32) + ch / 4] = (uint8_t)ke;
      ((uint8_t*)const_cast<float*>(a.c.v_scale))[sc * (D / 32) + ch / 4] = (uint8_t)ve;
    }
  } else if constexpr (KIND == kCacheInt8) {
    float x;
    v2u c;
    quantize8<D, BF16>(kx, &x, &c);
    *reinterpret_cast<v2u*>((uint8_t*)a.c.k + kd + 8 * ch) = c;
    if (ch == 0) const_cast<float*>(a.c.k_scale)[sc] = x;
    quantize8<D, BF16>(vx, &x, &c);
    *reinterpret_cast<v2u*>((uint8_t*)a.c.v + vd + 8 * ch) = c;
    if (ch == 0) const_cast<float*>(a.c.v_scale)[sc] = x;
  } else {
    *reinterpret_cast<v4i*>((uint16_t*)a.c.k + kd + 8 * ch) = kx;
    *reinterpret_cast<v4i*>((uint16_t*)a.c.v + vd + 8 * ch) = vx;
  }
  if (!SLOTS && a.weights && ch == 0) a.weights[((size_t)s * a.c.Hkv + h) * a.wstride + at] = 0.0f;
}

template <int D, bool BF16, bool TILED>
static void launch_store_t(const Store& s, int kind, dim3 grid, hipStream_t st) {
  const dim3 block(256);
  if (!s.slots) hipLaunchKernelGGL((kv_store_kernel<D, BF16, kCacheFp4, false, TILED>), grid, block, 0, st, s);
  else if (kind == kCacheFp4) hipLaunchKernelGGL((kv_store_kernel<D, BF16, kCacheFp4, true, TILED>), grid, block, 0, st, s);
  else if (kind == kCacheInt8) hipLaunchKernelGGL((kv_store_kernel<D, BF16, kCacheInt8, true, TILED>), grid, block, 0, st, s);
  else hipLaunchKernelGGL((kv_store_kernel<D, BF16, kCache16, true, TILED>), grid, block, 0, st, s);
}
// Rows in tiles, unless a sequence and head has too few of them for one.
template <int D, bool BF16>
static void launch_store(const Store& s, int kind, hipStream_t st) {
  const int per = 256 / (D / 8);
  if (s.a.N >= per) {
    launch_store_t<D, BF16, true>(s, kind, dim3((unsigned)cdiv(s.a.N, per), (unsigned)s.a.c.Hkv, (unsigned)s.a.c.S), st);
  } else {
    const long long rows = (long long)s.a.c.S * s.a.c.Hkv * s.a.N;
    launch_store_t<D, BF16, false>(s, kind, dim3((unsigned)((rows + per - 1) / per)), st);
  }
}
hipError_t launch_kv_store(const Append& a, const int64_t* slots, int D, bool bf16, int kind, hipStream_t st) {
  const Store s{a, slots, divide_by(a.c.Hkv * a.N), divide_by(a.N), divide_by(a.c.page_size)};
  if (D == 128) {
    if (bf16) launch_store<128, true>(s, kind, st);
    else launch_store<128, false>(s, kind, st);
  } else {
    if (bf16) launch_store<64, true>(s, kind, st);
    else launch_store<64, false>(s, kind, st);
  }
  return hipGetLastError();
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
template <int RB, typename Scale>                        // bytes of a row; what holds its scales
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
      Scale *ks = (Scale*)const_cast<float*>(a.c.k_scale), *vs = (Scale*)const_cast<float*>(a.c.v_scale);
      ks[di] = ks[si];
      vs[di] = vs[si];
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

hipError_t launch_kv_evict(const Evict& x, int D, bool fp4, hipStream_t st) {
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
  const int elem = a.c.k_scale ? 1 : 2, rb = fp4 ? D / 2 : D * elem, per = 256 / (rb / 16);
  const dim3 grid((unsigned)imin(cdiv(a.budget, per), imax(1, (int)(8192 / ((long long)a.c.S * a.c.Hkv)))),
                  (unsigned)a.c.Hkv, (unsigned)a.c.S);
  // (a row's scales move as one word: one in fp32, or 4 or 2 bytes of an MXFP4 row)
  if (rb == 256) hipLaunchKernelGGL((evict_move_kernel<256, uint32_t>), grid, dim3(256), 0, st, a, elem);
  else if (rb == 128) hipLaunchKernelGGL((evict_move_kernel<128, uint32_t>), grid, dim3(256), 0, st, a, elem);
  else if (rb == 64) hipLaunchKernelGGL((evict_move_kernel<64, uint32_t>), grid, dim3(256), 0, st, a, elem);
  else hipLaunchKernelGGL((evict_move_kernel<32, uint16_t>), grid, dim3(256), 0, st, a, elem);
  return hipGetLastError();
}

}  // namespace sage
