// Attention with a causal sliding window and sinks for gfx950, forward: query i
// sees key j iff j <= i and (j > i - window or j < sinks), up to the sequence's
// length (window.h).  Grouped heads: query head h reads key head h Hkv / Hq.
//   S^T (keys x queries) = K . Q^T,   online softmax in fp32,
//   O^T (dims x queries) += V^T . P^T,   O = O / l,   L = m + log l
// on v_mfma_f32_32x32x16 in the input's type.  4 waves x 32 queries per
// workgroup, 64-key tiles of K and V double-buffered in LDS, the operand layouts
// of the bf16 kernel (attn_bf16.hip).  Only the tiles that hold a key some query
// of the workgroup sees are loaded -- the sinks' and the window's -- and a wave
// computes only those that its own 32 queries see; scores are masked in the tiles
// on the diagonal and at the two edges of the window.
//
// Bound by issue: per 32 x 64 piece of D = 128 the 32 MFMAs take 1024 cycles of a SIMD,
// 32 exponentials 512 and the other VALU work about 400, and the two waves of a SIMD
// hide little of one kind under the other.  32768 tokens, 32/8 heads, window 4096:
// 2.20-2.26 ms a call, 910-940 TFLOP/s (a large bf16 matrix product: 1200).
//
// P is rounded to the input's type for the second product (relative error 2^-8
// in bf16, 2^-11 in fp16 per probability); everything else is fp32.
#include "bf16_tile.h"
#include "lm_args.h"
#include "mma16.h"
#include "window.h"

namespace sage {

// A probability of 0 times a value that is no finite number would be NaN, so a
// masked key's V could reach rows that do not see it.  Rather than look at every
// tile, the kernel looks at its result: a workgroup whose O holds anything but finite
// numbers runs its tiles again with V's infinities and NaN taken out and added where
// they are seen (split_nonfinite).

constexpr int WK = 64;         // keys per tile
constexpr int WW = 4;          // waves per workgroup (32 queries each)

// x with 0 for infinities and NaN; 1.0 in `pos` for +inf and NaN, in `neg` for -inf and NaN.
template <bool BF16>
__device__ __forceinline__ void split_nonfinite(const v4i x, v4i& fin, v4i& pos, v4i& neg) {
  constexpr uint32_t EXP = BF16 ? 0x7F80u : 0x7C00u, ONE = BF16 ? 0x3F80u : 0x3C00u;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint32_t f = 0, p = 0, n = 0;
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
      const uint32_t h = ((uint32_t)x[d] >> s) & 0xFFFFu;
      const bool bad = (h & EXP) == EXP, nan = bad && (h & 0x7FFFu) != EXP;
      if (!bad) f |= h << s;
      if (nan || (bad && !(h & 0x8000u))) p |= ONE << s;
      if (nan || (bad && (h & 0x8000u))) n |= ONE << s;
    }
    fin[d] = (int)f; pos[d] = (int)p; neg[d] = (int)n;
  }
}

// KG: groups of WW waves that take the tiles in turn and are joined at the end.
template <int D, bool BF16, int KG>
__global__ __launch_bounds__(64 * WW * KG, 2 / KG) void window_fwd_kernel(const WindowFwd a) {
  constexpr int NKS = D / 16, NDB = D / 32;
  constexpr float LAZY = 8.0f, SHIFT = BF16 ? 0.0f : kPShift<false> - LAZY;   // fp16: P at most 2^15 all the same
  static_assert(WK == 64, "a tile is two 32-key pieces");
  constexpr int ROW = D * 2, CH = ROW / 16, TB = WK * ROW;
  constexpr int GROUP = 4 * TB;                          // two stages of a K tile and a V tile per group of waves
  __shared__ __attribute__((aligned(256))) uint8_t lds[KG * GROUP];
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = KG == 1 ? wid : wid % WW, kg = KG == 1 ? 0 : wid / WW, lgroup = kg * GROUP;
  const int col = lane & 31, hi = lane >> 5;
  const int nqt = cdiv(a.N, 32 * WW);

  const unsigned lin = xcd_order(blockIdx.x, gridDim.x, a.B * a.Hkv);
  const int bh = (int)(lin / nqt), b = bh / a.Hq, h = bh - b * a.Hq, hk = h / (a.Hq / a.Hkv);
  const int qt = nqt - 1 - (int)(lin % nqt);                     // the longest rows first
  const int q0 = qt * (32 * WW), qw = q0 + wave * 32, qi = qw + col;
  const int n = a.lens ? cached_len(a.lens[b], a.N) : a.N;

  uint16_t* const orow = (uint16_t*)a.o + (b * a.os.b + h * a.os.h + (long long)qi * a.os.n);
  float* const lrow = a.lse ? a.lse + (size_t)bh * a.N + qi : nullptr;

  const int W = a.window, sinks = a.sinks;
  const int q1 = min(q0 + 32 * WW, n);                           // past the last query
  const TileList tl = q0 < n ? tile_list(q0 - W + 1, q1, sinks, WK) : TileList{0, 0, 0};

  v4i qreg[NKS];
  {
    const int qr = max(0, min(qi, n - 1));
    const uint16_t* q = (const uint16_t*)a.q + (b * a.qs.b + h * a.qs.h + (long long)qr * a.qs.n);
#pragma unroll
    for (int s = 0; s < NKS; ++s) qreg[s] = *reinterpret_cast<const v4i*>(q + 16 * s + 8 * hi);
  }

  // Tile loads as in attn_bf16.hip, with the rows' stride; rows past n read zero.
  constexpr int JR = 1024 / ROW, NJ = WK / JR, JW = NJ / WW;
  static_assert(NJ % WW == 0, "every wave loads the same number of pieces");
  static_assert(WW * JR % 16 == 0 || D == 64, "a lane's pieces have the same swizzle");
  static_assert(WW * JR % 32 == 0 || D == 128, "a lane's pieces have the same swizzle");
  const uint32_t kst = (uint32_t)(a.ks.n * 2), vst = (uint32_t)(a.vs.n * 2);
  const int jr = wave * JR + lane / CH;
  const uint32_t klo = jr * kst + bswz<CH>(jr, lane % CH) * 16, vlo = jr * vst + vswz<D>(jr, lane % CH) * 16;
  const uint8_t* kbase = (const uint8_t*)a.k + 2 * (b * a.ks.b + hk * a.ks.h);
  const uint8_t* vbase = (const uint8_t*)a.v + 2 * (b * a.vs.b + hk * a.vs.h);
  auto issue = [&](int kb, int stage) {
    uint8_t* L = lds + lgroup + stage * 2 * TB;
    const uint32_t rows = (uint32_t)min(n - kb, WK);
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(kbase + (size_t)kb * kst, (rows - 1) * kst + ROW);
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(vbase + (size_t)kb * vst, (rows - 1) * vst + ROW);
    const uint32_t k0 = opaque(klo), v0 = opaque(vlo);
#pragma unroll
    for (int i = 0; i < JW; ++i) {
      buf_load16(rk, k0 + WW * JR * i * kst, 0u, L + (wave + WW * i) * 1024);
      buf_load16(rv, v0 + WW * JR * i * vst, 0u, L + TB + (wave + WW * i) * 1024);
    }
  };

  const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const uint32_t rat = row_at<D, true>(), tat = tr_at<D>();

  v16f oacc[NDB];
  float m, l;
  // NS 32-key pieces of the tile at stage, from its row `off` on, key kb; hide0 / hide1: not that one
  auto piece = [&](auto NS_, auto CAREFUL_, int stage, int off, int kb, bool hide0, bool hide1) {
    constexpr int NS = decltype(NS_)::value;
    constexpr bool CAREFUL = decltype(CAREFUL_)::value != 0;
    const uint32_t L = l0 + lgroup + stage * 2 * TB + off * ROW;  // (32 rows on, the swizzle is the same)
    v16f sacc[NS];
    {
      const uint32_t ra = opaque(L + rat);
      if (NS == 2 && !hide0 && !hide1) {                 // the two halves in turn: neither waits for its own last result
        sacc[0] = sacc[NS - 1] = v16f{};
#pragma unroll
        for (int s = 0; s < NKS; ++s) {
          sacc[0] = mma32<BF16>(lds16(ra ^ (32 * s)), qreg[s], sacc[0]);
          sacc[NS - 1] = mma32<BF16>(lds16((ra ^ (32 * s)) + 32 * ROW), qreg[s], sacc[NS - 1]);
        }
        // four reads in front of the product that takes the first of them (the compiler alone reads,
        // waits and multiplies in turn; 681 -> 668 us on 4 x 4096 tokens)
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int s = 0; s < 2 * NKS; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (s + 4 < 2 * NKS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      } else {
#pragma unroll
        for (int t = 0; t < NS; ++t) {
          v16f acc = v16f{};
          if (!(t ? hide1 : hide0)) {
#pragma unroll
            for (int s = 0; s < NKS; ++s) acc = mma32<BF16>(lds16((ra ^ (32 * s)) + 32 * t * ROW), qreg[s], acc);
            __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
            for (int s = 0; s < NKS; ++s) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              if (s + 3 < NKS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
          }
          sacc[t] = acc;
        }
      }
    }
    if (kb + 32 * NS - 1 > qw || kb + 32 * NS > n || (kb <= qw + 31 - W && kb + 32 * NS > sinks)) {
      // element (t, e) is key kb + 4 hi + c with c = 32t + 8 (e >> 2) + (e & 3), kept iff
      // c < rem and (c >= low or c < sk): a sign mask selects its bits or those of -inf
      // (a minimum with -inf would let the NaN of a masked key through)
      const int base = kb + 4 * hi, rem = min(n, qi + 1) - base, low = qi - W + 1 - base, sk = sinks - base;
#pragma unroll
      for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int c = 32 * t + 8 * (e >> 2) + (e & 3);
          const uint32_t keep = (uint32_t)(((c - rem) & ~((c - low) & ~(c - sk))) >> 31);
          sacc[t][e] = __uint_as_float((__float_as_uint(sacc[t][e]) & keep) | (0xFF800000u & ~keep));
        }
    }
    float x = sacc[0][0];
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
      for (int e = (t == 0 ? 1 : 0); e < 16; ++e) x = smax(x, sacc[t][e]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float m_new = smax(m, smax(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
    // The sums are rescaled only when some row's maximum has grown by more than 2^LAZY
    // (a row's first key always has): until then its probabilities are up to 2^LAZY
    // larger.  Of 32 rows one has a new maximum in most of the first 30 tiles.
    if (__builtin_amdgcn_ballot_w64((m_new - m) * a.c2 > LAZY) != 0) {
      // (a row that has seen no key yet keeps m = -inf: 0 in its place is as good)
      const float alpha = __builtin_amdgcn_exp2f(m * a.c2 - (m_new == -INFINITY ? 0.0f : m_new * a.c2));   // 0 the first time
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[db][e] *= alpha;
    }
    // against 0 the probabilities of a row that has seen no key are 0, not NaN
    const float mp = (m == -INFINITY ? 0.0f : m * a.c2) - SHIFT;
    const uint32_t va = opaque(L + TB + tat);
    float ps[2] = {0.0f, 0.0f};
    static_for<2 * NS>([&](auto U_) {
      constexpr int u = decltype(U_)::value, t = u >> 1, base = 8 * (u & 1);
      if (t ? hide1 : hide0) return;
      v8bf vt[NDB];
      constexpr int OFF = 16 * u * ROW, OFF8 = OFF + 8 * ROW;
      if constexpr (NDB == 4) vt_read4<OFF, OFF8>(va, va ^ 64, va ^ 128, va ^ 192, vt[0], vt[1], vt[2], vt[3]);
      else vt_read2<OFF, OFF8>(va, va ^ 64, vt[0], vt[1]);
      v4i pk;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][base + 2 * i], a.c2, -mp));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][base + 2 * i + 1], a.c2, -mp));
        ps[i & 1] += p0;
        ps[i & 1] += p1;
        pk[i] = (int)pack16<BF16>(p0, p1);
      }
      if constexpr (CAREFUL) {
        v4i see;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          see[i] = (int)pack16<BF16>(sacc[t][base + 2 * i] == -INFINITY ? 0.0f : 1.0f, sacc[t][base + 2 * i + 1] == -INFINITY ? 0.0f : 1.0f);
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          v4i fin, pos, neg;
          __builtin_amdgcn_sched_barrier(0);             // one block's operands at a time: registers
          split_nonfinite<BF16>(__builtin_bit_cast(v4i, vt[db]), fin, pos, neg);
          oacc[db] = mma32<BF16>(fin, pk, oacc[db]);
          v16f c = mma32<BF16>(pos, see, v16f{});
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] += c[e] > 0.0f ? INFINITY : 0.0f;
          c = mma32<BF16>(neg, see, v16f{});
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] -= c[e] > 0.0f ? INFINITY : 0.0f;
        }
      } else {
#pragma unroll
        for (int db = 0; db < NDB; ++db) oacc[db] = mma32<BF16>(__builtin_bit_cast(v4i, vt[db]), pk, oacc[db]);
      }
    });
    l += ps[0] + ps[1];
  };
  auto attend = [&](auto CAREFUL_) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = v16f{};
    m = -INFINITY, l = 0.0f;

    if (kg < tl.count) issue(tl.tile(kg) * WK, 0);
    // The queries' registers are waited for here, behind the first tile's loads: left to their first
    // use, the compiler waits inside the loop, and for the tile in flight too (4 x 32 heads of 4096
    // tokens: 667 -> 630 us).
#pragma unroll
    for (int s = 0; s < NKS; ++s) asm volatile("" : "+v"(qreg[s]));
    for (int i = 0; i * KG < tl.count; ++i) {
      const int j = i * KG + kg, stage = i & 1;
      __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): this wave's loads of tile j have landed
      lds_barrier();                                     // everyone's; every wave is past the tile before
      if (j + KG < tl.count) issue(tl.tile(j + KG) * WK, stage ^ 1);
      if (KG > 1 && j >= tl.count) continue;
      const int kb = tl.tile(j) * WK;
      // a half is hidden if it lies past the wave's last query, or before its first query's window
      // and behind the sinks
      const bool hide0 = kb > qw + 31 || (kb + 32 <= qw - W + 1 && kb >= sinks);
      const bool hide1 = kb + 32 > qw + 31 || (kb + 64 <= qw - W + 1 && kb + 32 >= sinks);
      if (hide0 && hide1) continue;
      // D = 128: both halves in one softmax step, their scores computed in turn (2.29 -> 2.23 ms on
      // 32768 tokens, window 4096, against a half after the other).  D = 64: a step for each, as
      // 40 registers less are worth more than the shared step (54 -> 50 us on 8192 tokens, window 256).
      if constexpr (D == 64) {
#pragma unroll 1
        for (int t = 0; t < 2; ++t)
          if (!(t ? hide1 : hide0)) piece(ic<1>{}, CAREFUL_, stage, 32 * t, kb + 32 * t, false, false);
      } else {
        piece(ic<2>{}, CAREFUL_, stage, 0, kb, hide0, hide1);
      }
    }
  };
  attend(ic<0>{});
  bool odd = false;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) odd |= !(__builtin_fabsf(oacc[db][e]) < INFINITY);
  if (__syncthreads_or(odd)) attend(ic<1>{});          // (a barrier: every wave is past its last tile's LDS)

  if constexpr (KG == 2) {
    // the second group's sums join the first's of the same queries
    float* const x = reinterpret_cast<float*>(lds) + wave * (NDB * 16 + 2) * 64 + lane;
    __syncthreads();
    if (kg == 1) {
      x[0] = m;
      x[64] = l;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[(2 + db * 16 + e) * 64] = oacc[db][e];
    }
    __syncthreads();
    if (kg == 1) return;
    const float m1 = x[0], mm = smax(m, m1), mc = mm == -INFINITY ? 0.0f : mm * a.c2;
    const float f0 = __builtin_amdgcn_exp2f(m * a.c2 - mc), f1 = __builtin_amdgcn_exp2f(m1 * a.c2 - mc);
    m = mm;
    l = l * f0 + x[64] * f1;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[db][e] = oacc[db][e] * f0 + x[(2 + db * 16 + e) * 64] * f1;
  }
  if (qi >= a.N) return;
  const float ltot = l + __shfl_xor(l, 32, 64);
  // rows behind the sequence's end (their accumulators follow a copy of its last query) are 0 and -inf
  const bool live = qi < n;
  const float inv = live ? 1.0f / ltot : 0.0f;
  if (lrow && hi == 0)
    *lrow = live ? (m * a.c2 + (__builtin_log2f(ltot) - SHIFT)) * 0.69314718055994530942f : -INFINITY;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint32_t w0 = pack16<BF16>(oacc[db][4 * g] * inv, oacc[db][4 * g + 1] * inv);
      const uint32_t w1 = pack16<BF16>(oacc[db][4 * g + 2] * inv, oacc[db][4 * g + 3] * inv);
      *reinterpret_cast<v2u*>(orow + 32 * db + 8 * g + 4 * hi) = live ? v2u{w0, w1} : v2u{0u, 0u};
    }
}

template <int D, bool BF16>
static hipError_t launch_window_fwd_t(const WindowFwd& a, hipStream_t st) {
  // With a workgroup per CU or less, two groups of waves share its tiles (2 x 12 heads of
  // 1000 tokens, D = 64, causal: 23 -> 17.5 us, dQ 27 -> 22); with more, a second workgroup does.
  const long long blocks = (long long)cdiv(a.N, 32 * WW) * a.B * a.Hq;
  if (blocks <= 256) hipLaunchKernelGGL((window_fwd_kernel<D, BF16, 2>), dim3((unsigned)blocks), dim3(128 * WW), 0, st, a);
  else hipLaunchKernelGGL((window_fwd_kernel<D, BF16, 1>), dim3((unsigned)blocks), dim3(64 * WW), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_window_fwd(const WindowFwd& a, int D, bool bf16, hipStream_t st) {
  if (D == 128) return bf16 ? launch_window_fwd_t<128, true>(a, st) : launch_window_fwd_t<128, false>(a, st);
  return bf16 ? launch_window_fwd_t<64, true>(a, st) : launch_window_fwd_t<64, false>(a, st);
}

}  // namespace sage
