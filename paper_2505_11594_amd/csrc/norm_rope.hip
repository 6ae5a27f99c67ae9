// Norm of every query and key head with the rotation by position, and its backward, for
// gfx950.  Per row x of D channels, with weights w and angles t_i = p f_i of position p:
//   r = (mean(x^2) + eps)^-1/2,  y = x r w,  (z_a, z_b) = (y_a cos - y_b sin, y_b cos + y_a sin)
// where pair i < R / 2 is channels (i, i + R / 2) or (2i, 2i + 1); channels from R on are y.
// Backward, with g = the pairs of dz turned back and u = g w:
//   dw = sum over rows of g x r,   dx = r u - x r^3 mean(u x).
//
// D / 8 lanes hold a row, 8 channels each: four whole pairs, so nothing is exchanged but the
// sums.  A wave takes a token (or a part of its heads): its lanes find the token's angles
// once, one each, for all of its rows.  The bytes bound it: 32768 tokens of 32 / 8 heads, D = 128,
// take 133 us, 5.05 TB/s (a large copy: 5.27); 8192 tokens 34 us, their backward 51 and 4.8 for the
// weights' sums (VALU busy half of the time in all three).  The scalar registers that do not do lie in
// lanes of vector ones (4 in the forward, 23-25 in the backward): read per token, not in the loop over
// its rows.
//
// Angles: p f in 64 bits (a position has up to 31 bits, f 24: 53 keep the product's
// fraction of a turn to 2^-22 of one at the farthest), reduced there to an eighth of a turn
// around a quarter; sine and cosine by their series up to x^9 and x^10, whose rests are below
// 2^-29 there.
#include "lm_args.h"
#include "mma16.h"
#include "window.h"

namespace sage {

// x + its value in the lanes that a DPP control names.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
// Sum over the D / 8 lanes of a row; every lane gets the same bits.
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  x = add_dpp<0xB1>(x);                                  // lane ^ 1, ^ 2 within four
  x = add_dpp<0x4E>(x);
  x = add_dpp<0x141>(x);                                 // mirrored within eight
  if constexpr (D == 128) x = add_dpp<0x140>(x);         // mirrored within sixteen
  return x;
}

__device__ __forceinline__ void turn(int p, float f, float* cosine, float* sine) {
  const double t = (double)p * (double)f * 0.15915494309189533577;   // turns
  const double q = __builtin_rint(4.0 * t);
  const float x = (float)(t - 0.25 * q) * 6.28318530717958647692f;
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
  s = __builtin_fmaf(x2, s, 8.33333333e-3f);
  s = __builtin_fmaf(x2, s, -1.66666667e-1f);
  s = __builtin_fmaf(x * x2, s, x);
  float c = __builtin_fmaf(x2, -2.75573192e-7f, 2.48015873e-5f);
  c = __builtin_fmaf(x2, c, -1.38888889e-3f);
  c = __builtin_fmaf(x2, c, 4.16666667e-2f);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.0f);
  const int quarter = (int)(q - 4.0 * __builtin_floor(0.25 * q));    // 0 to 3
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  *cosine = quarter == 1 || quarter == 2 ? -a : a;
  *sine = quarter >= 2 ? -b : b;
}

// A lane's place in a row: channels c0 .. c0 + 3 and c1 .. c1 + 3.
template <bool PAIRS>
__device__ __forceinline__ void lane_channels(int l, int R, int* c0, int* c1) {
  const bool halves = !PAIRS && l < R / 8;
  *c0 = halves ? 4 * l : 8 * l;
  *c1 = halves ? R / 2 + 4 * l : 8 * l + 4;
}

struct Row8 {
  v2u a, b;
};
template <bool PAIRS>
__device__ __forceinline__ Row8 load_row(const uint16_t* x, int c0, int c1) {
  if constexpr (PAIRS) {
    const v4i v = *reinterpret_cast<const v4i*>(x + c0);
    return Row8{v2u{(uint32_t)v[0], (uint32_t)v[1]}, v2u{(uint32_t)v[2], (uint32_t)v[3]}};
  } else {
    return Row8{*reinterpret_cast<const v2u*>(x + c0), *reinterpret_cast<const v2u*>(x + c1)};
  }
}
template <bool PAIRS>
__device__ __forceinline__ void store_row(uint16_t* x, int c0, int c1, const Row8& r) {
  if constexpr (PAIRS) {
    *reinterpret_cast<v4i*>(x + c0) = v4i{(int)r.a[0], (int)r.a[1], (int)r.b[0], (int)r.b[1]};
  } else {
    *reinterpret_cast<v2u*>(x + c0) = r.a;
    *reinterpret_cast<v2u*>(x + c1) = r.b;
  }
}
template <bool BF16>
__device__ __forceinline__ void widen_row(const Row8& r, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[2 * i] = widen<BF16>((uint16_t)r.a[i]);
    x[2 * i + 1] = widen<BF16>((uint16_t)(r.a[i] >> 16));
    x[4 + 2 * i] = widen<BF16>((uint16_t)r.b[i]);
    x[5 + 2 * i] = widen<BF16>((uint16_t)(r.b[i] >> 16));
  }
}
template <bool BF16>
__device__ __forceinline__ Row8 pack_row(const float* x) {
  return Row8{v2u{pack16<BF16>(x[0], x[1]), pack16<BF16>(x[2], x[3])}, v2u{pack16<BF16>(x[4], x[5]), pack16<BF16>(x[6], x[7])}};
}
// The four pairs turned by +angle, or by -angle.
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void turn_row(float* x, const float* cs, const float* sn) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float& a = x[PAIRS ? 2 * j : j];
    float& b = x[PAIRS ? 2 * j + 1 : 4 + j];
    const float s = BACK ? -sn[j] : sn[j], a0 = a;
    a = __builtin_fmaf(a0, cs[j], -(b * s));
    b = __builtin_fmaf(b, cs[j], a0 * s);
  }
}

// A wave's token.
struct Token {
  int b, n, p;
  bool inside;                                           // not behind the sequence's end
};
__device__ __forceinline__ Token find_token(const NormRope& a, int tk) {
  Token t;
  t.b = tk / a.N;
  t.n = tk - t.b * a.N;
  t.inside = !a.lens || t.n < a.lens[t.b];
  t.p = t.n;
  if (a.pos) t.p = a.pos_each ? a.pos[tk] : (int)((unsigned)a.pos[t.b] + (unsigned)t.n);
  return t;
}
// Cosines and sines of this lane's pairs; freq: inv_freq of pair `lane`.
template <int D>
__device__ __forceinline__ void token_angles(const NormRope& a, int p, float freq, float* cs, float* sn) {
  const int l = (threadIdx.x & 63) % (D / 8);
  float c, s;
  turn(p, freq, &c, &s);
#pragma unroll
  for (int j = 0; j < 4; ++j) {                          // pair 4 l + j; channels that are not rotated: angle 0
    const int from = 4 * l + j;
    cs[j] = __shfl(c, from & 63, 64);
    sn[j] = __shfl(s, from & 63, 64);
    if (from >= a.R / 2) { cs[j] = 1.0f; sn[j] = 0.0f; }
  }
}

__device__ __forceinline__ void load_weight(const float* w, int c0, int c1, float* out) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    out[j] = w ? w[c0 + j] : 1.0f;
    out[4 + j] = w ? w[c1 + j] : 1.0f;
  }
}

// A token's rows, in steps of 512 / D rows that a wave takes at once: first q's, then k's.  A wave
// whose part of them is `part` of split takes the steps part, part + split, ...
struct Step {
  bool q, ok;                                            // ok: this lane has a row (else it holds the last one again)
  int h;
};
template <int D>
__device__ __forceinline__ Step step_of(const NormRope& a, int i, int sq) {
  constexpr int RPW = 512 / D;
  const int rg = (threadIdx.x & 63) / (D / 8);
  Step s;
  s.q = i < sq;
  const int H = s.q ? a.Hq : a.Hkv, h = (s.q ? i : i - sq) * RPW + rg;
  s.ok = h < H;
  s.h = imin(h, H - 1);
  return s;
}
__device__ __forceinline__ const uint16_t* row_in(const void* x, const Strides& s, const Token& t, int h) {
  return (const uint16_t*)x + (t.b * s.b + t.n * s.n) + h * s.h;
}
__device__ __forceinline__ uint16_t* row_out(void* x, const Strides& s, const Token& t, int h) {
  return (uint16_t*)x + (t.b * s.b + t.n * s.n) + h * s.h;
}

// Steps whose rows are on their way behind those at work.  (4948 tokens of 48 heads, D = 64: 13.9
// us; 14.7 with 1, 15.2 with 3 or 4, whose registers let fewer waves on a SIMD.)
constexpr int NU = 2;
template <int D, bool BF16, bool PAIRS>
__global__ __launch_bounds__(256) void norm_rope_fwd_kernel(const NormRope a) {
  constexpr int RPW = 512 / D;
  const int lane = threadIdx.x & 63, l = lane % (D / 8);
  int c0, c1;
  lane_channels<PAIRS>(l, a.R, &c0, &c1);
  float wq[8], wk[8];
  load_weight(a.wq, c0, c1, wq);
  load_weight(a.wk, c0, c1, wk);
  const float freq = lane < a.R / 2 ? a.freq[lane] : 0.0f;
  const int waves = a.B * a.N * a.split, sq = cdiv(a.Hq, RPW), steps = sq + cdiv(a.Hkv, RPW);
  for (long long wv = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); wv < waves;
       wv += (long long)gridDim.x * 4) {
    const int tk = (int)wv / a.split, part = (int)wv - tk * a.split;
    const Token t = find_token(a, tk);
    if (!t.inside) {
      for (int i = part; i < steps; i += a.split) {
        const Step s = step_of<D>(a, i, sq);
        if (s.ok) store_row<PAIRS>(row_out(s.q ? a.zq : a.zk, s.q ? a.zqs : a.zks, t, s.h), c0, c1, Row8{});
      }
      continue;
    }
    Row8 in[NU];
    auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
        if (i0 + u * a.split < steps) {
          const Step s = step_of<D>(a, i0 + u * a.split, sq);
          in[u] = load_row<PAIRS>(row_in(s.q ? a.q : a.k, s.q ? a.qs : a.ks, t, s.h), c0, c1);
        }
    };
    load(part);                                          // (the angles are found meanwhile)
    float cs[4], sn[4];
    token_angles<D>(a, t.p, freq, cs, sn);
    for (int i0 = part; i0 < steps; i0 += NU * a.split) {
      Row8 cur[NU];
#pragma unroll
      for (int u = 0; u < NU; ++u) cur[u] = in[u];
      load(i0 + NU * a.split);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        if (i0 + u * a.split >= steps) break;
        const Step s = step_of<D>(a, i0 + u * a.split, sq);
        float v[8], ss = 0.0f;
        widen_row<BF16>(cur[u], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<D>(ss), 1.0f / D, a.eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r * (s.q ? wq[i] : wk[i]);
        turn_row<PAIRS, false>(v, cs, sn);
        if (s.ok) store_row<PAIRS>(row_out(s.q ? a.zq : a.zk, s.q ? a.zqs : a.zks, t, s.h), c0, c1, pack_row<BF16>(v));
      }
    }
  }
}

// Gradients of x, and per workgroup the sums for those of the weights: part [workgroups][q, k][D].
constexpr int BU = 2;
template <int D, bool BF16, bool PAIRS>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(const NormRope a) {
  constexpr int LPR = D / 8, RPW = 64 / LPR;
  __shared__ float sums[4][2][D];
  const int lane = threadIdx.x & 63, l = lane % LPR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int c0, c1;
  lane_channels<PAIRS>(l, a.R, &c0, &c1);
  float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
  load_weight(a.wq, c0, c1, wq);
  load_weight(a.wk, c0, c1, wk);
  const float freq = lane < a.R / 2 ? a.freq[lane] : 0.0f;
  const int waves = a.B * a.N * a.split, sq = cdiv(a.Hq, RPW), steps = sq + cdiv(a.Hkv, RPW);
  for (long long wv = (long long)blockIdx.x * 4 + wave; wv < waves; wv += (long long)gridDim.x * 4) {
    const int tk = (int)wv / a.split, part = (int)wv - tk * a.split;
    const Token t = find_token(a, tk);
    if (!t.inside) {
      for (int i = part; i < steps; i += a.split) {
        const Step s = step_of<D>(a, i, sq);
        if (s.ok) store_row<PAIRS>(row_out(s.q ? a.zq : a.zk, s.q ? a.zqs : a.zks, t, s.h), c0, c1, Row8{});
      }
      continue;
    }
    Row8 in[BU], gin[BU];
    auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < BU; ++u)
        if (i0 + u * a.split < steps) {
          const Step s = step_of<D>(a, i0 + u * a.split, sq);
          in[u] = load_row<PAIRS>(row_in(s.q ? a.q : a.k, s.q ? a.qs : a.ks, t, s.h), c0, c1);
          gin[u] = load_row<PAIRS>(row_in(s.q ? a.gq : a.gk, s.q ? a.gqs : a.gks, t, s.h), c0, c1);
        }
    };
    load(part);
    float cs[4], sn[4];
    token_angles<D>(a, t.p, freq, cs, sn);
    for (int i0 = part; i0 < steps; i0 += BU * a.split) {
      Row8 cur[BU], gcur[BU];
#pragma unroll
      for (int u = 0; u < BU; ++u) { cur[u] = in[u]; gcur[u] = gin[u]; }
      load(i0 + BU * a.split);
#pragma unroll
      for (int u = 0; u < BU; ++u) {
        if (i0 + u * a.split >= steps) break;
        const Step s = step_of<D>(a, i0 + u * a.split, sq);
        if (!s.ok) cur[u] = gcur[u] = Row8{};            // adds nothing to the weights' gradients
        float v[8], d[8], ss = 0.0f, ux = 0.0f;
        widen_row<BF16>(cur[u], v);
        widen_row<BF16>(gcur[u], d);
        turn_row<PAIRS, true>(d, cs, sn);
        const auto rows = [&](const float* w, float* dw) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            ss = __builtin_fmaf(v[i], v[i], ss);
            ux = __builtin_fmaf(d[i] * w[i], v[i], ux);
          }
          const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<D>(ss), 1.0f / D, a.eps));
          const float m = row_sum<D>(ux) * (1.0f / D) * r * r;       // mean(u x) r^2
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dw[i] = __builtin_fmaf(d[i], v[i] * r, dw[i]);
            d[i] = r * __builtin_fmaf(-m, v[i], d[i] * w[i]);
          }
        };
        if (s.q) rows(wq, dwq);
        else rows(wk, dwk);
        if (s.ok) store_row<PAIRS>(row_out(s.q ? a.zq : a.zk, s.q ? a.zqs : a.zks, t, s.h), c0, c1, pack_row<BF16>(d));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
      dwq[i] += __shfl_xor(dwq[i], o, 64);
      dwk[i] += __shfl_xor(dwk[i], o, 64);
    }
    const int c = i < 4 ? c0 + i : c1 + i - 4;
    if (lane < LPR) {
      sums[wave][0][c] = dwq[i];
      sums[wave][1][c] = dwk[i];
    }
  }
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const float* s = &sums[0][0][threadIdx.x];
    a.part[(size_t)blockIdx.x * 2 * D + threadIdx.x] = (s[0] + s[2 * D]) + (s[4 * D] + s[6 * D]);
  }
}

// The workgroups' sums added up: a workgroup per 16 channels of q's or k's weights, 64 threads
// to a channel's parts.
template <int D>
__global__ __launch_bounds__(1024) void weight_sum_kernel(const float* part, int blocks, float* dwq, float* dwk) {
  __shared__ float sums[64][17];
  const int c = threadIdx.x & 15, y = threadIdx.x >> 4, at = blockIdx.x * 16 + c;
  float x = 0.0f;
  for (int i0 = y; i0 < blocks; i0 += 16 * 64) {         // 16 loads on their way
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = part[(size_t)imin(i0 + 64 * u, blocks - 1) * 2 * D + at];
#pragma unroll
    for (int u = 0; u < 16; ++u) x += i0 + 64 * u < blocks ? v[u] : 0.0f;
  }
  sums[y][c] = x;
  __syncthreads();
  for (int o = 32; o >= 1; o >>= 1) {
    if (y < o) sums[y][c] += sums[y + o][c];
    __syncthreads();
  }
  float* out = at < D ? dwq : dwk;
  if (y == 0 && out) out[at < D ? at : at - D] = sums[0][c];
}

// Waves that share a token's heads: one, and more where the tokens do not fill the GPU, up to
// one per step.  A wave's start -- its weights, its token, the angles -- takes as long as several
// steps, so that 4 waves on each of 1024 SIMDs do (4948 tokens of 48 heads, D = 64: 13.9 us, 16.6
// with 8, 25 with 16; of 40 heads, D = 128: 22.5, 24, 30).
static int split_of(long long tokens, int Hq, int Hkv, int D) {
  const int rpw = 512 / D, steps = cdiv(Hq, rpw) + cdiv(Hkv, rpw);
  int split = 1;
  while (split * 2 <= steps && tokens * split < 4096) split *= 2;
  return split;
}
// The backward's workgroups: each leaves a sum of its own, so no more than fill the GPU once at 4
// waves per SIMD.  That is what the kernel's 124 registers let run, but for fp16 in pairs: its 132 let 3,
// and a quarter of the workgroups comes in a second round (8192 tokens of 32 / 8 heads, D = 128, graph of
// calls: 61 us; fp16 in halves 53, bf16 in pairs 56 and in halves 53-54.  2 x 1000 of 12 / 4, D = 64: 15.3;
// 12.8, 13.8 and 12.7).
int norm_rope_bwd_blocks(long long tokens, int Hq, int Hkv, int D) {
  const long long want = (tokens * split_of(tokens, Hq, Hkv, D) + 3) / 4;
  return (int)(want < 1024 ? want : 1024);
}

template <int D, bool BF16>
static void launch_t(const NormRope& a, bool pairs, bool bwd, unsigned blocks, hipStream_t st) {
  if (!bwd) {
    if (pairs) hipLaunchKernelGGL((norm_rope_fwd_kernel<D, BF16, true>), dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_rope_fwd_kernel<D, BF16, false>), dim3(blocks), dim3(256), 0, st, a);
  } else {
    if (pairs) hipLaunchKernelGGL((norm_rope_bwd_kernel<D, BF16, true>), dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_rope_bwd_kernel<D, BF16, false>), dim3(blocks), dim3(256), 0, st, a);
  }
}
hipError_t launch_norm_rope(const NormRope& args, int D, bool bf16, bool pairs, bool bwd, hipStream_t st) {
  NormRope a = args;
  const long long tokens = (long long)a.B * a.N;
  a.split = split_of(tokens, a.Hq, a.Hkv, D);
  const long long want = (tokens * a.split + 3) / 4;
  const unsigned blocks = bwd ? (unsigned)norm_rope_bwd_blocks(tokens, a.Hq, a.Hkv, D) : (unsigned)(want < 1 << 20 ? want : 1 << 20);
  if (D == 128) {
    if (bf16) launch_t<128, true>(a, pairs, bwd, blocks, st);
    else launch_t<128, false>(a, pairs, bwd, blocks, st);
  } else {
    if (bf16) launch_t<64, true>(a, pairs, bwd, blocks, st);
    else launch_t<64, false>(a, pairs, bwd, blocks, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !bwd || (!a.dwq && !a.dwk)) return e;
  if (D == 128) hipLaunchKernelGGL(weight_sum_kernel<128>, dim3(16), dim3(1024), 0, st, a.part, (int)blocks, a.dwq, a.dwk);
  else hipLaunchKernelGGL(weight_sum_kernel<64>, dim3(8), dim3(1024), 0, st, a.part, (int)blocks, a.dwq, a.dwk);
  return hipGetLastError();
}

}  // namespace sage
