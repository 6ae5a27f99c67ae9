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

template <int D, bool BF16>
__global__ __launch_bounds__(64 * WW, 2) void window_fwd_kernel(const WindowFwd a) {
  constexpr int NSUB = WK / 32, NKS = D / 16, NPK = WK / 16, NDB = D / 32;
  constexpr int ROW = D * 2, CH = ROW / 16, TB = WK * ROW;
  __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TB];   // two stages of a K tile and a V tile
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hi = lane >> 5;
  const int nqt = cdiv(a.N, 32 * WW);

  // Each XCD takes a run of neighbouring tiles: they share keys, and heads of a group follow each other.
  const unsigned total = gridDim.x, xcd = blockIdx.x & 7;
  const unsigned lin = xcd * (total >> 3) + min(xcd, total & 7u) + (blockIdx.x >> 3);
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
  uint32_t klo[JW], vlo[JW];
  const uint32_t kst = (uint32_t)(a.ks.n * 2), vst = (uint32_t)(a.vs.n * 2);
#pragma unroll
  for (int i = 0; i < JW; ++i) {
    const int r = (wave + WW * i) * JR + lane / CH;
    klo[i] = r * kst + bswz<CH>(r, lane % CH) * 16;
    vlo[i] = r * vst + vswz<D>(r, lane % CH) * 16;
  }
  const uint8_t* kbase = (const uint8_t*)a.k + 2 * (b * a.ks.b + hk * a.ks.h);
  const uint8_t* vbase = (const uint8_t*)a.v + 2 * (b * a.vs.b + hk * a.vs.h);
  auto issue = [&](int kb, int stage) {
    uint8_t* L = lds + stage * 2 * TB;
    const uint32_t rows = (uint32_t)min(n - kb, WK);
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(kbase + (size_t)kb * kst, (rows - 1) * kst + ROW);
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(vbase + (size_t)kb * vst, (rows - 1) * vst + ROW);
#pragma unroll
    for (int i = 0; i < JW; ++i) {
      buf_load16(rk, klo[i], 0u, L + (wave + WW * i) * 1024);
      buf_load16(rv, vlo[i], 0u, L + TB + (wave + WW * i) * 1024);
    }
  };

  uint32_t vo[NDB];
  {
    const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int r = 4 * hi + (lane & 15) / 4, c0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
    for (int db = 0; db < NDB; ++db) vo[db] = l0 + TB + r * ROW + vswz<D>(r, 4 * db + c0) * 16 + 8 * (lane & 1);
  }

  v16f oacc[NDB];
  float m, l;
  auto attend = [&](auto CAREFUL_) {
    constexpr bool CAREFUL = decltype(CAREFUL_)::value != 0;
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = v16f{};
    m = -INFINITY, l = 0.0f;

    if (tl.count > 0) issue(tl.tile(0) * WK, 0);
    for (int j = 0; j < tl.count; ++j) {
      __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): this wave's loads of tile j have landed
      __syncthreads();                                   // everyone's; every wave is past tile j - 1
      if (j + 1 < tl.count) issue(tl.tile(j + 1) * WK, (j + 1) & 1);
      const uint8_t* L = lds + (j & 1) * 2 * TB;
      const int kb = tl.tile(j) * WK;
      // keys past the wave's last query, or before its first query's window and behind the sinks
      if (kb > qw + 31 || (kb + WK <= qw - W + 1 && kb >= sinks)) continue;
      v16f sacc[NSUB];
#pragma unroll
      for (int t = 0; t < NSUB; ++t) {
        const int row = 32 * t + col;
        v16f acc = v16f{};
#pragma unroll
        for (int s = 0; s < NKS; ++s) {
          const v4i x = *reinterpret_cast<const v4i*>(L + row * ROW + bswz<CH>(row, 2 * s + hi) * 16);
          acc = mma32<BF16>(x, qreg[s], acc);
        }
        sacc[t] = acc;
      }
      if (kb + WK - 1 > qw || kb + WK > n || (kb <= qw + 31 - W && kb + WK > sinks)) {
        // element (t, e) is key kb + 4 hi + c with c = 32t + 8 (e >> 2) + (e & 3), kept iff
        // c < rem and (c >= low or c < sk): a sign mask selects its bits or those of -inf
        // (a minimum with -inf would let the NaN of a masked key through)
        const int base = kb + 4 * hi, rem = min(n, qi + 1) - base, low = qi - W + 1 - base, sk = sinks - base;
#pragma unroll
        for (int t = 0; t < NSUB; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int c = 32 * t + 8 * (e >> 2) + (e & 3);
            const uint32_t keep = (uint32_t)(((c - rem) & ~((c - low) & ~(c - sk))) >> 31);
            sacc[t][e] = __uint_as_float((__float_as_uint(sacc[t][e]) & keep) | (0xFF800000u & ~keep));
          }
      }
      float x = sacc[0][0];
#pragma unroll
      for (int t = 0; t < NSUB; ++t)
#pragma unroll
        for (int e = (t == 0 ? 1 : 0); e < 16; ++e) x = smax(x, sacc[t][e]);
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      const float m_new = smax(m, smax(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
      // a row that has seen no key yet keeps m = -inf: against 0 its probabilities are 0, not NaN
      const float mc = m_new == -INFINITY ? 0.0f : m_new * a.c2;
      const float alpha = __builtin_amdgcn_exp2f(m * a.c2 - mc);    // 0 on the first tile
      m = m_new;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] *= alpha;
      }
      const float mp = mc - kPShift<BF16>;
      uint32_t va[NDB];
#pragma unroll
      for (int db = 0; db < NDB; ++db) va[db] = vo[db] + (uint32_t)((j & 1) * 2 * TB);
      float ps[2] = {0.0f, 0.0f};
      static_for<NPK>([&](auto U_) {
        constexpr int u = decltype(U_)::value, t = u >> 1, base = 8 * (u & 1);
        v8bf vt[NDB];
        constexpr int OFF = 16 * u * ROW, OFF8 = OFF + 8 * ROW;
        if constexpr (NDB == 4) vt_read4<OFF, OFF8>(va[0], va[1], va[2], va[3], vt[0], vt[1], vt[2], vt[3]);
        else vt_read2<OFF, OFF8>(va[0], va[1], vt[0], vt[1]);
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
            __builtin_amdgcn_sched_barrier(0);           // one block's operands at a time: registers
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
      l = l * alpha + (ps[0] + ps[1]);
    }
  };
  attend(ic<0>{});
  bool odd = false;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) odd |= !(__builtin_fabsf(oacc[db][e]) < INFINITY);
  if (__syncthreads_or(odd)) attend(ic<1>{});          // (a barrier: every wave is past its last tile's LDS)

  if (qi >= a.N) return;
  const float ltot = l + __shfl_xor(l, 32, 64);
  // rows behind the sequence's end (their accumulators follow a copy of its last query) are 0 and -inf
  const bool live = qi < n;
  const float inv = live ? 1.0f / ltot : 0.0f;
  if (lrow && hi == 0)
    *lrow = live ? (m * a.c2 + (__builtin_log2f(ltot) - kPShift<BF16>)) * 0.69314718055994530942f : -INFINITY;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint32_t w0 = pack16<BF16>(oacc[db][4 * g] * inv, oacc[db][4 * g + 1] * inv);
      const uint32_t w1 = pack16<BF16>(oacc[db][4 * g + 2] * inv, oacc[db][4 * g + 3] * inv);
      *reinterpret_cast<v2u*>(orow + 32 * db + 8 * g + 4 * hi) = live ? v2u{w0, w1} : v2u{0u, 0u};
    }
}

hipError_t launch_window_fwd(const WindowFwd& a, int D, bool bf16, hipStream_t st) {
  const dim3 grid((unsigned)((long long)cdiv(a.N, 32 * WW) * a.B * a.Hq)), block(64 * WW);
  if (D == 128) {
    if (bf16) hipLaunchKernelGGL((window_fwd_kernel<128, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((window_fwd_kernel<128, false>), grid, block, 0, st, a);
  } else {
    if (bf16) hipLaunchKernelGGL((window_fwd_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((window_fwd_kernel<64, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sage
