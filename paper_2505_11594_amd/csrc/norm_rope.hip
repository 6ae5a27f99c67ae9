// Norm of every query and key head with the rotation by position, and its backward, for
// gfx950.  Per row x of D channels, with weights w and angles t_i = p f_i of position p:
//   r = (mean(x^2) + eps)^-1/2,  y = x r w,  (z_a, z_b) = (y_a cos - y_b sin, y_b cos + y_a sin)
// where pair i < R / 2 is channels (i, i + R / 2) or (2i, 2i + 1); channels from R on are y.
// Backward, with g = the pairs of dz turned back and u = g w:
//   dw = sum over rows of g x r,   dx = r u - x r^3 mean(u x).
//
// D / 8 lanes hold a row, 8 channels each: four whole pairs, so nothing is exchanged but the
// sums.  A wave takes a token (or a part of its heads): its lanes find the token's angles
// once, one each, for all of its rows.  The bytes bound it.
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

// A wave's token and its angles; false where there is none.
struct Token {
  int b, n;
  bool inside;                                           // not behind the sequence's end
  float cs[4], sn[4];                                    // of this lane's pairs
};
template <int D>
__device__ __forceinline__ void find_token(const NormRope& a, long long tk, Token& t) {
  const int lane = threadIdx.x & 63, l = lane % (D / 8);
  t.b = (int)(tk / a.N);
  t.n = (int)(tk - (long long)t.b * a.N);
  t.inside = !a.lens || t.n < a.lens[t.b];
  int p = t.n;
  if (a.pos) p = a.pos_each ? a.pos[tk] : (int)((unsigned)a.pos[t.b] + (unsigned)t.n);
  float c, s;
  turn(p, lane < a.R / 2 ? a.freq[lane] : 0.0f, &c, &s);
#pragma unroll
  for (int j = 0; j < 4; ++j) {                          // pair 4 l + j; channels that are not rotated: angle 0
    const int from = 4 * l + j;
    t.cs[j] = __shfl(c, from & 63, 64);
    t.sn[j] = __shfl(s, from & 63, 64);
    if (from >= a.R / 2) { t.cs[j] = 1.0f; t.sn[j] = 0.0f; }
  }
}

__device__ __forceinline__ void load_weight(const float* w, int c0, int c1, float* out) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    out[j] = w ? w[c0 + j] : 1.0f;
    out[4 + j] = w ? w[c1 + j] : 1.0f;
  }
}

constexpr int NU = 4;                                    // row loads in flight per lane

// A token's heads of q or k, those of this wave's part.  One wave step is 512 / D rows.
template <int D, bool BF16, bool PAIRS>
__device__ __forceinline__ void fwd_heads(const NormRope& a, const Token& t, const void* x, void* z, const Strides& xs,
                                          const Strides& zs, int H, int first, const float* w, int c0, int c1) {
  constexpr int LPR = D / 8, RPW = 64 / LPR;
  const int rg = (threadIdx.x & 63) / LPR;
  const uint16_t* src = (const uint16_t*)x + t.b * xs.b + t.n * xs.n;
  uint16_t* dst = (uint16_t*)z + t.b * zs.b + t.n * zs.n;
  for (int h0 = first * RPW; h0 < H; h0 += NU * a.split * RPW) {
    Row8 in[NU];
    if (t.inside) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
        in[u] = load_row<PAIRS>(src + imin(h0 + u * a.split * RPW + rg, H - 1) * xs.h, c0, c1);
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int h = h0 + u * a.split * RPW + rg;
      float v[8] = {};
      if (t.inside) {
        widen_row<BF16>(in[u], v);
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<D>(ss), 1.0f / D, a.eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r * w[i];
        turn_row<PAIRS, false>(v, t.cs, t.sn);
      }
      if (h < H) store_row<PAIRS>(dst + h * zs.h, c0, c1, pack_row<BF16>(v));
    }
  }
}

template <int D, bool BF16, bool PAIRS>
__global__ __launch_bounds__(256) void norm_rope_fwd_kernel(const NormRope a) {
  constexpr int LPR = D / 8, RPW = 64 / LPR;
  const int l = threadIdx.x % LPR;
  int c0, c1;
  lane_channels<PAIRS>(l, a.R, &c0, &c1);
  float wq[8], wk[8];
  load_weight(a.wq, c0, c1, wq);
  load_weight(a.wk, c0, c1, wk);
  const long long tokens = (long long)a.B * a.N;
  const int sq = cdiv(a.Hq, RPW);
  for (long long i = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < tokens * a.split;
       i += (long long)gridDim.x * 4) {
    const long long tk = i / a.split;
    const int part = (int)(i - tk * a.split);
    Token t;
    find_token<D>(a, tk, t);
    // steps of q, then of k, dealt out to the token's waves in turn
    fwd_heads<D, BF16, PAIRS>(a, t, a.q, a.zq, a.qs, a.zqs, a.Hq, part, wq, c0, c1);
    const int over = sq % a.split;
    fwd_heads<D, BF16, PAIRS>(a, t, a.k, a.zk, a.ks, a.zks, a.Hkv, part >= over ? part - over : part + a.split - over, wk, c0, c1);
  }
}

template <int D, bool BF16, bool PAIRS>
__device__ __forceinline__ void bwd_heads(const NormRope& a, const Token& t, const void* x, const void* g, void* dx,
                                          const Strides& xs, const Strides& gs, const Strides& ds, int H, int first,
                                          const float* w, float* dw, int c0, int c1) {
  constexpr int LPR = D / 8, RPW = 64 / LPR, U = NU / 2;
  const int rg = (threadIdx.x & 63) / LPR;
  const uint16_t* src = (const uint16_t*)x + t.b * xs.b + t.n * xs.n;
  const uint16_t* gsrc = (const uint16_t*)g + t.b * gs.b + t.n * gs.n;
  uint16_t* dst = (uint16_t*)dx + t.b * ds.b + t.n * ds.n;
  for (int h0 = first * RPW; h0 < H; h0 += U * a.split * RPW) {
    Row8 in[U], gin[U];
    if (t.inside) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = imin(h0 + u * a.split * RPW + rg, H - 1);
        in[u] = load_row<PAIRS>(src + h * xs.h, c0, c1);
        gin[u] = load_row<PAIRS>(gsrc + h * gs.h, c0, c1);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * a.split * RPW + rg;
      float v[8] = {}, d[8] = {};
      if (t.inside) {
        if (h >= H) in[u] = gin[u] = Row8{};             // (a lane without a row holds the last one's)
        widen_row<BF16>(in[u], v);
        widen_row<BF16>(gin[u], d);
        turn_row<PAIRS, true>(d, t.cs, t.sn);
        float ss = 0.0f, ux = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          ss = __builtin_fmaf(v[i], v[i], ss);
          ux = __builtin_fmaf(d[i] * w[i], v[i], ux);
        }
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row_sum<D>(ss), 1.0f / D, a.eps));
        const float m = row_sum<D>(ux) * (1.0f / D) * r * r;         // mean(u x) r^2
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dw[i] = __builtin_fmaf(d[i], v[i] * r, dw[i]);
          d[i] = r * __builtin_fmaf(-m, v[i], d[i] * w[i]);
        }
      }
      if (h < H) store_row<PAIRS>(dst + h * ds.h, c0, c1, pack_row<BF16>(d));
    }
  }
}

// Gradients of x, and per workgroup the sums for those of the weights: part [workgroups][q, k][D].
template <int D, bool BF16, bool PAIRS>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(const NormRope a) {
  constexpr int LPR = D / 8, RPW = 64 / LPR;
  __shared__ float sums[4][2][D];
  const int lane = threadIdx.x & 63, l = threadIdx.x % LPR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int c0, c1;
  lane_channels<PAIRS>(l, a.R, &c0, &c1);
  float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
  load_weight(a.wq, c0, c1, wq);
  load_weight(a.wk, c0, c1, wk);
  const long long tokens = (long long)a.B * a.N;
  const int sq = cdiv(a.Hq, RPW);
  for (long long i = (long long)blockIdx.x * 4 + wave; i < tokens * a.split; i += (long long)gridDim.x * 4) {
    const long long tk = i / a.split;
    const int part = (int)(i - tk * a.split);
    Token t;
    find_token<D>(a, tk, t);
    bwd_heads<D, BF16, PAIRS>(a, t, a.q, a.gq, a.zq, a.qs, a.gqs, a.zqs, a.Hq, part, wq, dwq, c0, c1);
    const int over = sq % a.split;
    bwd_heads<D, BF16, PAIRS>(a, t, a.k, a.gk, a.zk, a.ks, a.gks, a.zks, a.Hkv,
                              part >= over ? part - over : part + a.split - over, wk, dwk, c0, c1);
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
#pragma unroll 4
  for (int i = y; i < blocks; i += 64) x += part[(size_t)i * 2 * D + at];
  sums[y][c] = x;
  __syncthreads();
  for (int o = 32; o >= 1; o >>= 1) {
    if (y < o) sums[y][c] += sums[y + o][c];
    __syncthreads();
  }
  float* out = at < D ? dwq : dwk;
  if (y == 0 && out) out[at < D ? at : at - D] = sums[0][c];
}

// Waves that share a token's heads: one, and more where the tokens do not fill the GPU (8
// waves on each of 1024 SIMDs), up to one per step.
static int split_of(long long tokens, int Hq, int Hkv, int D) {
  const int rpw = 512 / D, steps = cdiv(Hq, rpw) + cdiv(Hkv, rpw);
  int split = 1;
  while (split * 2 <= steps && tokens * split < 8192) split *= 2;
  return split;
}
// The backward's workgroups: each leaves a sum of its own, so no more than fill the GPU twice.
int norm_rope_bwd_blocks(long long tokens, int Hq, int Hkv, int D) {
  const long long want = (tokens * split_of(tokens, Hq, Hkv, D) + 3) / 4;
  return (int)(want < 2048 ? want : 2048);
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
