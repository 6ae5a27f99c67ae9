// Backward pass of the window attention (attn_window.hip) for gfx950.  With
// P = exp(S / sqrt(D) - L), delta_i = sum_d dO_i O_i and dS = P o (dO V^T - delta):
//   dV_j = sum_i P_ij dO_i,   dK_j = sum_i dS_ij Q_i / sqrt(D),   dQ_i = sum_j dS_ij K_j / sqrt(D)
// summed over the query heads of a group for dK and dV, in fp32 and in a fixed order.
//
// Two passes over the visible pairs, each recomputing S and dP: dkv_kernel (4
// products; a wave holds 32 keys' K, V, dK^T and dV^T in registers and walks the
// queries that see them, all heads of the group) and dq_kernel (3 products; a wave
// holds 32 queries and walks their keys).  One pass would need dQ added up across
// workgroups: atomics whose order changes the result, or a stored dS, whose 4 bytes
// per pair (written and read) take longer than the two products they save.
//
// A query tile (or key tile) lies in LDS once, in a layout that serves both the row
// reads of S and dP and the transposing reads of the second products (vswz); P and dS
// stay in registers, as in the forward.  MFMA issue and LDS reads (32 KiB per 32
// products of 32 x 32 x 16) bound both kernels.
//
// Sink keys are seen by every later query, 32768 / 1152 times as many as others of a
// long sequence: dkv_kernel leaves them out, a launch of its SINK form takes them in
// chunks of queries and join_sinks_kernel adds the chunks.
//
// P and dS are rounded to the input's type for the second products.  In fp16 both
// carry a power of two that keeps them normal numbers: P 2^15, and dS the largest
// with which 2 max|dO_i| max|V_j| (a bound of |dP - delta|, over the group's heads)
// stays below 2^15.
#include "bf16_tile.h"
#include "lm_args.h"
#include "mma16.h"
#include "window.h"

namespace sage {

constexpr int BT = 64;                  // rows of a tile in LDS
constexpr int PR = 64;                  // rows per workgroup of the row pass
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ int seq_len(const WindowBwd& a, int b) { return a.lens ? cached_len(a.lens[b], a.N) : a.N; }
// Rows of a sequence's lb and delta arrays.
__device__ __forceinline__ int row_pad(int N) { return (N + BT - 1) / BT * BT; }

// lb = -L log2(e) (and P's power of two; -inf behind the sequence's end: P = 0 there)
// and -delta per query row, as the kernels add them; in fp16 also the largest |dO_i|
// (and, from blockIdx.y >= B Hq on, |V_j|) of every PR rows.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void rows_kernel(const WindowBwd a) {
  constexpr int LPR = D / 8, RPP = 256 / LPR, PASSES = PR / RPP;   // lanes per row, rows per pass
  __shared__ float red[4];
  const int tid = threadIdx.x, ch = tid % LPR;
  const int nb = cdiv(a.N, PR);
  const bool vrows = (int)blockIdx.y >= a.B * a.Hq;
  const int bh = vrows ? blockIdx.y - a.B * a.Hq : blockIdx.y, H = vrows ? a.Hkv : a.Hq;
  const int b = bh / H, h = bh - b * H, n = seq_len(a, b);
  const Strides& xs = vrows ? a.vs : a.gs;
  const uint16_t* x = (const uint16_t*)(vrows ? a.v : a.dout) + b * xs.b + h * xs.h + 8 * ch;
  const Strides& ys = vrows ? a.vs : a.os;
  const uint16_t* y = vrows ? x : (const uint16_t*)a.o + b * a.os.b + h * a.os.h + 8 * ch;
  // every load in front, behind no branch (24 heads of 1000 tokens, D = 64: 5.4 -> 4.3 us); rows
  // past the end take the last one and count as zero
  v4i xr[PASSES], yr[PASSES];
  float lse[PASSES];
#pragma unroll
  for (int r = 0; r < PASSES; ++r) {
    const int i = imax(0, imin(blockIdx.x * PR + r * RPP + tid / LPR, n - 1));
    xr[r] = *reinterpret_cast<const v4i*>(x + i * xs.n);
    yr[r] = *reinterpret_cast<const v4i*>(y + i * ys.n);
    lse[r] = a.lse[(size_t)bh * a.N + i];               // (of V's rows, which are no more, not used)
  }
  float most = 0.0f;
#pragma unroll
  for (int r = 0; r < PASSES; ++r) {
    const int i = blockIdx.x * PR + r * RPP + tid / LPR;
    float dot = 0.0f, sq = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float gv = widen<BF16>((uint16_t)((uint32_t)xr[r][e / 2] >> (16 * (e & 1))));
      dot = __builtin_fmaf(gv, widen<BF16>((uint16_t)((uint32_t)yr[r][e / 2] >> (16 * (e & 1)))), dot);
      if constexpr (!BF16) sq = __builtin_fmaf(gv, gv, sq);
    }
    if (i >= n) dot = sq = 0.0f;
#pragma unroll
    for (int s = LPR / 2; s >= 1; s >>= 1) {
      dot += __shfl_xor(dot, s, 64);
      if constexpr (!BF16) sq += __shfl_xor(sq, s, 64);
    }
    if (!vrows && ch == 0) {                             // (the arrays hold whole tiles of rows)
      const size_t at = (size_t)bh * row_pad(a.N) + i;
      a.delta[at] = -dot;
      a.lb[at] = i < n ? kPShift<BF16> - lse[r] * kLog2e : -INFINITY;
    }
    most = __builtin_fmaxf(most, sq);
  }
  if constexpr (!BF16) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, s, 64));
    if ((tid & 63) == 0) red[tid >> 6] = most;
    __syncthreads();
    if (tid == 0)
      a.norms[(size_t)blockIdx.y * nb + blockIdx.x] =
          __builtin_sqrtf(__builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3])));
  }
}
static_assert(PR == BT, "the row pass fills whole tiles of rows");

// The power of two that dS of each (sequence, key head) carries in fp16, from the norms of
// its row blocks: one workgroup each.  If every wave of the kernels behind looked through
// the norms itself, G N / 64 of them, a window's constant work per workgroup would grow with N
// (fp16 step of 16 / 1 heads, D = 64, window 64: 32768 tokens 488 -> 258 us with this
// launch, 2048 tokens 59 -> 57.5, 2 x 12 / 4 heads of 1000 tokens 78 either way).
constexpr int SW = 16;                  // waves
__global__ __launch_bounds__(64 * SW) void scale_kernel(const WindowBwd a) {
  __shared__ float red[2][SW];
  const int b = blockIdx.x / a.Hkv, hk = blockIdx.x - b * a.Hkv, tid = threadIdx.x, nb = cdiv(a.N, PR), G = a.Hq / a.Hkv;
  const float* g = a.norms + ((size_t)b * a.Hq + hk * G) * nb;
  const float* v = a.norms + ((size_t)a.B * a.Hq + b * a.Hkv + hk) * nb;
  float gm = 0.0f, vm = 0.0f;
#pragma unroll 4
  for (int i = tid; i < G * nb; i += 64 * SW) gm = __builtin_fmaxf(gm, g[i]);
#pragma unroll 4
  for (int i = tid; i < nb; i += 64 * SW) vm = __builtin_fmaxf(vm, v[i]);
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    gm = __builtin_fmaxf(gm, __shfl_xor(gm, s, 64));
    vm = __builtin_fmaxf(vm, __shfl_xor(vm, s, 64));
  }
  if ((tid & 63) == 0) {
    red[0][tid >> 6] = gm;
    red[1][tid >> 6] = vm;
  }
  __syncthreads();
  if (tid > 0) return;
#pragma unroll
  for (int w = 1; w < SW; ++w) {
    gm = __builtin_fmaxf(gm, red[0][w]);
    vm = __builtin_fmaxf(vm, red[1][w]);
  }
  const float bound = 2.0f * gm * vm;
  int e = 15;
  if (bound > 0.0f && bound < INFINITY) __builtin_frexpf(bound, &e);   // bound < 2^e
  a.scales[blockIdx.x] = __builtin_ldexpf(1.0f, imax(-100, imin(100, 15 - e)));
}
template <bool BF16>
__device__ __forceinline__ float ds_scale(const WindowBwd& a, int b, int hk) {
  return BF16 ? 1.0f : a.scales[(size_t)b * a.Hkv + hk];
}

// S and dP - delta: the 32 rows at `at` and TB bytes behind times the 32 columns of b and
// c, the second on top of g (-delta), the two products in turn (each alone would wait for its own last result, and its rows,
// all read ahead, would not leave enough registers for two waves per SIMD).
template <int D, bool BF16, int TB, int AHEAD = 3>
__device__ __forceinline__ void rows_times(uint32_t at, const v4i* b, const v4i* c, v16f& s, v16f& g) {
  s = v16f{};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    s = mma32<BF16>(lds16(at ^ (32 * i)), b[i], s);
    g = mma32<BF16>(lds16((at + TB) ^ (32 * i)), c[i], g);
  }
  // AHEAD reads in front of the product that takes the first of them (left alone, the
  // compiler reads, waits and multiplies in turn: 743 -> 727 us for a training step of 8192 tokens)
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + AHEAD < D / 8) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}
// The query tiles [t0, t1) of which some query sees one of the keys [k0, k0 + keys).
struct TileRange {
  int t0, t1;
};
__host__ __device__ __forceinline__ TileRange query_tiles(int k0, int keys, int n, int N, int window, bool sink) {
  TileRange r = {k0 / BT, k0 / BT};
  if (k0 < n) r.t1 = cdiv(sink ? n : imin(n, imin(N, k0 + keys - 1 + window)), BT);
  return r;
}

// One 32 x 32 block of (query, key) pairs for a wave that holds 32 keys (kreg, vreg;
// lane: key l % 32): adds to dv and dk (dims x keys).  The block's queries are rows
// [32 t, +32) of the tile at L (Q, then dO, then lb and delta).
template <int D, bool BF16>
__device__ __forceinline__ void dkv_block(uint32_t L, uint32_t rat, uint32_t tat, int t, const v4i* kreg, const v4i* vreg,
                                          v16f* dk, v16f* dv, float c2, float f15, bool mask, int first, int past) {
  constexpr int ROW = D * 2, TB = BT * ROW;
  const int hi = (threadIdx.x & 63) >> 5;
  const uint32_t ra = opaque(L + t * 32 * ROW + rat);
  // element e is query 32 t + 8 (e >> 2) + 4 hi + (e & 3) of the tile, visible iff first <= it < past
  const int at = 32 * t + 4 * hi;
  const uint32_t la = opaque(L + 2 * TB + 4 * at);
  v16f s, g;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const v4f dl = lds4f(la + 4 * BT + 32 * q);
#pragma unroll
    for (int e = 0; e < 4; ++e) g[4 * q + e] = dl[e];
  }
  rows_times<D, BF16, TB>(ra, kreg, vreg, s, g);
  if (mask) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int c = at + 8 * (e >> 2) + (e & 3);
      s[e] = c >= first && c < past ? s[e] : -INFINITY;
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const v4f lb = lds4f(la + 32 * q);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[4 * q + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * q + e], c2, lb[e]));
  }
  uint32_t pw[8], dw[8];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = s[4 * q + e] * (BF16 ? g[4 * q + e] : g[4 * q + e] * f15);
    pw[2 * q] = pack16<BF16>(s[4 * q], s[4 * q + 1]); pw[2 * q + 1] = pack16<BF16>(s[4 * q + 2], s[4 * q + 3]);
    dw[2 * q] = pack16<BF16>(d[0], d[1]); dw[2 * q + 1] = pack16<BF16>(d[2], d[3]);
  }
  const uint32_t ta = opaque(L + t * 32 * ROW + tat);
  static_for<2>([&](auto U_) {
    constexpr int u = decltype(U_)::value;
    const v4i pk = {(int)pw[4 * u], (int)pw[4 * u + 1], (int)pw[4 * u + 2], (int)pw[4 * u + 3]};
    const v4i dsk = {(int)dw[4 * u], (int)dw[4 * u + 1], (int)dw[4 * u + 2], (int)dw[4 * u + 3]};
    cols_times<D, BF16, TB + 16 * u * ROW>(ta, pk, dv);
    cols_times<D, BF16, 16 * u * ROW>(ta, dsk, dk);
  });
}

// dK and dV.  SINK: 2 waves share 32 sink keys and take one half of each query tile;
// else 4 waves x 32 keys.  Grid x: (sequence, key head) times the key blocks times
// the chunks of the blocks' query tiles (over all heads of the group), `share` tiles
// each; with more than one chunk their parts go to the workspace, in fp32.
template <int D, bool BF16, bool SINK>
__global__ __launch_bounds__(SINK ? 128 : 256, SINK ? 1 : 2) void dkv_kernel(const WindowBwd a) {
  constexpr int W = SINK ? 2 : 4;                        // waves
  constexpr int KB = SINK ? 32 : 128;                    // keys per workgroup
  constexpr int ROW = D * 2, CH = ROW / 16, TB = BT * ROW, NKS = D / 16, NDB = D / 32;
  constexpr int STAGE = 2 * TB + 2 * BT * 4;             // Q, dO, lb, delta
  static_assert(STAGE % 256 == 0, "addresses inside a tile are xor-ed");
  __shared__ __attribute__((aligned(256))) uint8_t lds[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hi = lane >> 5;
  const int nkb = SINK ? cdiv(a.sinks, KB) : cdiv(a.N, KB);
  unsigned lin = xcd_order(blockIdx.x, gridDim.x, a.B * a.Hkv);
  const int chunks = SINK ? a.chunks : a.mchunks, chunk = (int)(lin % chunks);
  lin /= chunks;
  const int bh = (int)(lin / nkb), b = bh / a.Hkv, hk = bh - b * a.Hkv, G = a.Hq / a.Hkv;
  const int k0 = (int)(lin % nkb) * KB, kw = SINK ? k0 : k0 + 32 * wave, key = kw + col;
  const int n = seq_len(a, b), Np = row_pad(a.N);

  // query tiles that see some of the keys, once per head of the group
  const TileRange tr = query_tiles(k0, KB, n, a.N, a.window, SINK);
  const int t0 = tr.t0, t1 = tr.t1, nt = t1 - t0;
  const int all = !SINK && k0 + KB <= a.sinks ? 0 : nt * G;      // (not for sink keys alone)
  const int share = SINK ? cdiv(all, chunks) : a.mshare;
  const int it0 = imin(all, chunk * share), it1 = imin(all, it0 + share);
  if (!SINK && chunk > 0 && it0 == it1) return;

  v4i kreg[NKS], vreg[NKS];
  {
    const int kr = imax(0, imin(key, n - 1));
    const uint16_t* k = (const uint16_t*)a.k + (b * a.ks.b + hk * a.ks.h + (long long)kr * a.ks.n);
    const uint16_t* v = (const uint16_t*)a.v + (b * a.vs.b + hk * a.vs.h + (long long)kr * a.vs.n);
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      kreg[s] = *reinterpret_cast<const v4i*>(k + 16 * s + 8 * hi);
      vreg[s] = *reinterpret_cast<const v4i*>(v + 16 * s + 8 * hi);
    }
  }
  const float f = ds_scale<BF16>(a, b, hk), f15 = f * 0x1p-15f;

  constexpr int JR = 1024 / ROW, NJ = BT / JR, JW = NJ / W;
  static_assert(W * JR % 8 == 0, "a lane's pieces have the same swizzle");
  const uint32_t qst = (uint32_t)(a.qs.n * 2), gst = (uint32_t)(a.gs.n * 2);
  const int jr = wave * JR + lane / CH;
  const uint32_t qlo = jr * qst + vswz<D>(jr, lane % CH) * 16, glo = jr * gst + vswz<D>(jr, lane % CH) * 16;
  auto issue = [&](int g, int tile, int stage) {
    uint8_t* L = lds + stage * STAGE;
    const int h = hk * G + g, qb = tile * BT;
    const uint32_t rows = (uint32_t)imin(n - qb, BT);
    const uint8_t* q = (const uint8_t*)a.q + 2 * (b * a.qs.b + h * a.qs.h) + (size_t)qb * qst;
    const uint8_t* o = (const uint8_t*)a.dout + 2 * (b * a.gs.b + h * a.gs.h) + (size_t)qb * gst;
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(q, (rows - 1) * qst + ROW), rg = make_rsrc(o, (rows - 1) * gst + ROW);
    const uint32_t q0 = opaque(qlo), g0 = opaque(glo);
#pragma unroll
    for (int i = 0; i < JW; ++i) {
      buf_load16(rq, q0 + W * JR * i * qst, 0u, L + (wave + W * i) * 1024);
      buf_load16(rg, g0 + W * JR * i * gst, 0u, L + TB + (wave + W * i) * 1024);
    }
    const size_t at = ((size_t)b * a.Hq + h) * Np + qb;
    if (wave == 0) buf_load4(make_rsrc(a.lb + at, BT * 4), 4 * lane, 0u, L + 2 * TB);
    if (wave == 1) buf_load4(make_rsrc(a.delta + at, BT * 4), 4 * lane, 0u, L + 2 * TB + BT * 4);
  };
  const uint32_t rat = row_at<D>(), tat = tr_at<D>();
  const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

  v16f dk[NDB], dv[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = v16f{};
  int g = nt > 0 ? it0 / nt : 0, tile = nt > 0 ? t0 + it0 % nt : 0;
  if (it0 < it1) issue(g, tile, 0);
  for (int it = it0; it < it1; ++it) {
    const int qb = tile * BT;
    if (++tile == t1) { tile = t0; ++g; }
    __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wave's loads of the tile have landed
    __syncthreads();                                     // everyone's; every wave is past the tile before
    const int st = (it - it0) & 1;
    if (it + 1 < it1) issue(g, tile, st ^ 1);
    const uint32_t L = l0 + st * STAGE;
    // queries [first, past) of the tile see this lane's key
    const int first = key - qb, past = SINK ? BT : key + a.window - qb;
    if constexpr (SINK) {
      if (qb + 32 * wave + 31 < kw) continue;
      dkv_block<D, BF16>(L, rat, tat, wave, kreg, vreg, dk, dv, a.c2, f15, qb + 32 * wave < kw + 31, first, past);
    } else {
#pragma unroll 1
      for (int t = 0; t < 2; ++t) {
        const int q0 = qb + 32 * t;
        if (q0 + 31 < kw || q0 >= kw + 31 + a.window) continue;
        dkv_block<D, BF16>(L, rat, tat, t, kreg, vreg, dk, dv, a.c2, f15, q0 < kw + 31 || q0 + 31 >= kw + a.window, first, past);
      }
    }
  }

  const float sv = BF16 ? 1.0f : 0x1p-15f, sk = a.rsd / f;
  if constexpr (SINK) {
    // add the two waves' sums; the chunk's part goes to the workspace
    __syncthreads();
    float* x = reinterpret_cast<float*>(lds);            // [2 D][32 keys] of wave 1
    if (wave == 1) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[((db * 16 + e) * 2) * 64 + lane] = dk[db][e];
          x[((db * 16 + e) * 2 + 1) * 64 + lane] = dv[db][e];
        }
    }
    __syncthreads();
    if (wave == 0) {
      float* part = a.part + ((((size_t)bh * nkb + k0 / KB) * a.chunks + chunk) * 2 * 32 + col) * D;
      const bool live = key < n;                         // keys behind the end were read as copies of the last
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v4f y, z;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = (db * 16 + 4 * q + e) * 2;
            y[e] = live ? (dk[db][4 * q + e] + x[r * 64 + lane]) * sk : 0.0f;
            z[e] = live ? (dv[db][4 * q + e] + x[(r + 1) * 64 + lane]) * sv : 0.0f;
          }
          *reinterpret_cast<v4f*>(part + 32 * db + 8 * q + 4 * hi) = y;
          *reinterpret_cast<v4f*>(part + 32 * D + 32 * db + 8 * q + 4 * hi) = z;
        }
    }
  } else {
    if (key >= a.N || key < a.sinks) return;             // the sinks' rows are join_sinks_kernel's
    const bool live = key < n;
    if (chunks > 1) {
      float* part = a.mpart + ((((size_t)bh * nkb + k0 / KB) * chunks + chunk) * 2 * KB + (key - k0)) * D;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v4f y, z;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = live ? dk[db][4 * q + e] * sk : 0.0f;
            z[e] = live ? dv[db][4 * q + e] * sv : 0.0f;
          }
          *reinterpret_cast<v4f*>(part + 32 * db + 8 * q + 4 * hi) = y;
          *reinterpret_cast<v4f*>(part + KB * D + 32 * db + 8 * q + 4 * hi) = z;
        }
      return;
    }
    uint16_t* kr = (uint16_t*)a.dk + ((size_t)bh * a.N + key) * D;
    uint16_t* vr = (uint16_t*)a.dv + ((size_t)bh * a.N + key) * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const v2u y = {pack16<BF16>(dk[db][4 * q] * sk, dk[db][4 * q + 1] * sk), pack16<BF16>(dk[db][4 * q + 2] * sk, dk[db][4 * q + 3] * sk)};
        const v2u z = {pack16<BF16>(dv[db][4 * q] * sv, dv[db][4 * q + 1] * sv), pack16<BF16>(dv[db][4 * q + 2] * sv, dv[db][4 * q + 3] * sv)};
        *reinterpret_cast<v2u*>(kr + 32 * db + 8 * q + 4 * hi) = live ? y : v2u{0u, 0u};
        *reinterpret_cast<v2u*>(vr + 32 * db + 8 * q + 4 * hi) = live ? z : v2u{0u, 0u};
      }
  }
}

// Sink keys' dK and dV from the chunks' parts, in their order: one workgroup per key,
// one thread per channel of dK and dV.
template <int D, bool BF16>
__global__ __launch_bounds__(2 * D) void join_sinks_kernel(const WindowBwd a) {
  const int bh = blockIdx.y, key = blockIdx.x, nkb = cdiv(a.sinks, 32), which = threadIdx.x / D, d = threadIdx.x % D;
  const float* p = a.part + ((((size_t)bh * nkb + key / 32) * a.chunks * 2 + which) * 32 + key % 32) * D + d;
  float x = 0.0f;
#pragma unroll 16
  for (int c = 0; c < a.chunks; ++c) x += p[(size_t)c * 2 * 32 * D];
  uint16_t* o = (uint16_t*)(which ? a.dv : a.dk) + ((size_t)bh * a.N + key) * D;
  o[d] = (uint16_t)pack16<BF16>(x, 0.0f);
}

// The other keys' dK and dV, where their query tiles were cut into chunks: 4 channels
// of one key per thread.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_keys_kernel(const WindowBwd a) {
  constexpr int KB = 128, TPK = D / 2;                   // threads per key: D / 4 for each of dK and dV
  const int bh = blockIdx.y, b = bh / a.Hkv, nkb = cdiv(a.N, KB);
  const int key = blockIdx.x * (256 / TPK) + threadIdx.x / TPK, x = threadIdx.x % TPK, which = x / (D / 4), d = x % (D / 4) * 4;
  if (key >= a.N || key < a.sinks) return;
  const TileRange tr = query_tiles(key / KB * KB, KB, seq_len(a, b), a.N, a.window, false);
  const int parts = imax(1, cdiv((tr.t1 - tr.t0) * (a.Hq / a.Hkv), a.mshare));
  const float* p = a.mpart + ((((size_t)bh * nkb + key / KB) * a.mchunks * 2 + which) * KB + key % KB) * D + d;
  v4f y = v4f{};
#pragma unroll 4
  for (int c = 0; c < parts; ++c) y += *reinterpret_cast<const v4f*>(p + (size_t)c * 2 * KB * D);
  uint16_t* o = (uint16_t*)(which ? a.dv : a.dk) + ((size_t)bh * a.N + key) * D + d;
  *reinterpret_cast<v2u*>(o) = v2u{pack16<BF16>(y[0], y[1]), pack16<BF16>(y[2], y[3])};
}

// dQ: 4 waves x 32 queries, the forward's walk over the key tiles.
//
// delta comes from O in 16 bits, so it is off by d_i = sum_d dO_i (O rounded - O), and
// every dS_ij by P_ij d_i: dQ would be off by d_i times the average key, which is
// large where keys share an offset, as trained models' do.  But sum_j dS_ij = 0, so
// any vector c may be taken off the keys: dQ_i = sum_j dS_ij K_j - c sum_j dS_ij,
// where the second sum holds the rounded dS that the product took.  c is the mean
// of the workgroup's last key tile.  (Error of dQ for keys N(0,1) with an N(0,1)
// offset per channel, 8192 tokens, window 1024, bf16: 3.7e-3 without c.)
// KG: groups of 4 waves that take the tiles in turn and are added at the end.
//
// Where a row sees few keys, |O| is as large as |V| and d_i as large as the rounding of
// dS itself.  Workgroups whose first row sees no more than EXACT keys (the first rows of
// a sequence; all under a short window) walk their tiles twice: the first time (2
// products) they add up sum_j P_ij (dP_ij - delta_i) in fp32, which is what delta is off
// by, and put it right for themselves and for dK and dV behind them.  (15 tokens, bf16:
// errors of dQ and dK 3.3e-3 -> 2.4e-3; their roundings alone give 2.3e-3.)  With more
// keys of like weight d_i is small against dS's rounding.  The second walk makes a training
// step of 8192 tokens, 32 / 8 heads, under a window of 128 10% longer (289 -> 318 us), of 256
// 13% (348 -> 393); windows above EXACT pay for their first rows alone (257: 345 -> 346).
constexpr int EXACT = 256;

template <int D, bool BF16, int KG>
__global__ __launch_bounds__(256 * KG, 2 / KG) void dq_kernel(const WindowBwd a) {
  constexpr int W = 4, ROW = D * 2, CH = ROW / 16, TB = BT * ROW, NKS = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(256))) uint8_t lds[KG * 4 * TB];   // two stages of a K tile and a V tile per group
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = KG == 1 ? wid : wid % W, kg = KG == 1 ? 0 : wid / W, lgroup = kg * 4 * TB;
  const int col = lane & 31, hi = lane >> 5;
  const int nqt = cdiv(a.N, 32 * W);
  const unsigned lin = xcd_order(blockIdx.x, gridDim.x, a.B * a.Hkv);
  const int bh = (int)(lin / nqt), b = bh / a.Hq, h = bh - b * a.Hq, hk = h / (a.Hq / a.Hkv);
  const int qt = nqt - 1 - (int)(lin % nqt), q0 = qt * (32 * W), qw = q0 + wave * 32, qi = qw + col;
  const int n = seq_len(a, b), win = a.window, sinks = a.sinks;
  const TileList tl = q0 < n ? tile_list(q0 - win + 1, imin(q0 + 32 * W, n), sinks, BT) : TileList{0, 0, 0};

  v4i qreg[NKS], greg[NKS];
  const int qr = imax(0, imin(qi, n - 1));
  {
    const uint16_t* q = (const uint16_t*)a.q + (b * a.qs.b + h * a.qs.h + (long long)qr * a.qs.n);
    const uint16_t* g = (const uint16_t*)a.dout + (b * a.gs.b + h * a.gs.h + (long long)qr * a.gs.n);
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      qreg[s] = *reinterpret_cast<const v4i*>(q + 16 * s + 8 * hi);
      greg[s] = *reinterpret_cast<const v4i*>(g + 16 * s + 8 * hi);
    }
  }
  const size_t at = ((size_t)b * a.Hq + h) * row_pad(a.N) + qr;
  const float lb = a.lb[at];
  v16f dl;                                               // -delta, where dP's sums start
#pragma unroll
  for (int e = 0; e < 16; ++e) dl[e] = a.delta[at];
  const float f = ds_scale<BF16>(a, b, hk), f15 = f * 0x1p-15f;

  constexpr int JR = 1024 / ROW, NJ = BT / JR, JW = NJ / W;
  static_assert(W * JR % 8 == 0, "a lane's pieces have the same swizzle");
  const uint32_t kst = (uint32_t)(a.ks.n * 2), vst = (uint32_t)(a.vs.n * 2);
  const int jr = wave * JR + lane / CH;
  const uint32_t klo = jr * kst + vswz<D>(jr, lane % CH) * 16, vlo = jr * vst + vswz<D>(jr, lane % CH) * 16;
  const uint8_t* kbase = (const uint8_t*)a.k + 2 * (b * a.ks.b + hk * a.ks.h);
  const uint8_t* vbase = (const uint8_t*)a.v + 2 * (b * a.vs.b + hk * a.vs.h);
  auto issue = [&](int kb, int stage) {
    uint8_t* L = lds + lgroup + stage * 2 * TB;
    const uint32_t rows = (uint32_t)imin(n - kb, BT);
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(kbase + (size_t)kb * kst, (rows - 1) * kst + ROW);
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(vbase + (size_t)kb * vst, (rows - 1) * vst + ROW);
    const uint32_t k0 = opaque(klo), v0 = opaque(vlo);
#pragma unroll
    for (int i = 0; i < JW; ++i) {
      buf_load16(rk, k0 + W * JR * i * kst, 0u, L + (wave + W * i) * 1024);
      buf_load16(rv, v0 + W * JR * i * vst, 0u, L + TB + (wave + W * i) * 1024);
    }
  };
  const uint32_t rat = row_at<D>(), tat = tr_at<D>();
  const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  v16f dq[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dq[db] = v16f{};
  float dsum = 0.0f;

  auto walk = [&](auto FIRST_) {
    constexpr bool FIRST = decltype(FIRST_)::value != 0;
    if (kg < tl.count) issue(tl.tile(kg) * BT, 0);
    for (int i = 0; i * KG < tl.count; ++i) {
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
      const int j = i * KG + kg;
      if (j + KG < tl.count) issue(tl.tile(j + KG) * BT, (i + 1) & 1);
      if (KG > 1 && j >= tl.count) continue;
      const uint32_t L = l0 + lgroup + (i & 1) * 2 * TB;
      const int kb = tl.tile(j) * BT;
      static_for<2>([&](auto T_) {
        constexpr int t = decltype(T_)::value;
        const int kt = kb + 32 * t;
        if (kt > qw + 31 || (kt + 32 <= qw - win + 1 && kt >= sinks)) return;
        const uint32_t ra = opaque(L + t * 32 * ROW + rat);
        v16f s, g = dl;
        rows_times<D, BF16, TB>(ra, qreg, greg, s, g);
        uint32_t dw[8];
        const bool mask = kt + 31 > qw || kt + 32 > n || (kt <= qw + 31 - win && kt + 32 > sinks);
        const int base = kt + 4 * hi, rem = imin(n, qi + 1) - base, low = qi - win + 1 - base, sk = sinks - base;
        float d[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c2, lb));
          d[e] = p * (BF16 ? g[e] : g[e] * f15);
        }
        if (mask) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int c = 8 * (e >> 2) + (e & 3);
            d[e] = __uint_as_float(__float_as_uint(d[e]) & (uint32_t)(((c - rem) & ~((c - low) & ~(c - sk))) >> 31));
          }
        }
        if constexpr (FIRST) {
#pragma unroll
          for (int e = 0; e < 16; ++e) dsum += d[e];
          return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dw[e] = pack16<BF16>(d[2 * e], d[2 * e + 1]);
          dsum = add_pair<BF16>(dw[e], dsum);
        }
        const uint32_t ta = opaque(L + tat);
        static_for<2>([&](auto U_) {
          constexpr int u = decltype(U_)::value;
          cols_times<D, BF16, (32 * t + 16 * u) * ROW>(ta, v4i{(int)dw[4 * u], (int)dw[4 * u + 1], (int)dw[4 * u + 2], (int)dw[4 * u + 3]}, dq);
        });
      });
    }
  };
  if (imin(q0 + 1, win) <= EXACT) {
    walk(ic<1>{});
    dsum += __shfl_xor(dsum, 32, 64);
    if constexpr (KG == 2) {
      float* const x = reinterpret_cast<float*>(lds) + wave * 32 + col;
      __syncthreads();
      if (hi == 0) x[kg * 128] = dsum;
      __syncthreads();
      dsum = x[0] + x[128];
    }
    __syncthreads();                                     // the tiles' LDS is free again
    dsum /= f;
#pragma unroll
    for (int e = 0; e < 16; ++e) dl[e] -= dsum;
    if (kg == 0 && hi == 0 && qi < n) a.delta[at] = dl[0];
    dsum = 0.0f;
  }
  walk(ic<0>{});
  // c: the mean of the last tile's keys, summed in 256 / (D / 2) groups of rows.  It lies in
  // its group's stage `last`; the sums go to that group's other stage.
  constexpr int NG = 512 / D;
  const int li = (tl.count - 1) / KG, lg = KG == 1 ? 0 : imax(0, tl.count - 1) % KG, last = li & 1;
  float* const sums = reinterpret_cast<float*>(lds + lg * 4 * TB + (last ^ 1) * 2 * TB);
  const int kl = tl.count > 0 ? tl.tile(tl.count - 1) * BT : 0;
  if (tl.count > 0 && tid < 256) {
    const uint8_t* L = lds + lg * 4 * TB + last * 2 * TB;
    const int ch = tid % (D / 2), g = tid / (D / 2);
    float x = 0.0f, y = 0.0f;
    for (int r = g; r < imin(n - kl, BT); r += NG) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(L + r * ROW + vswz<D>(r, ch / 4) * 16 + 4 * (ch % 4));
      x += widen<BF16>((uint16_t)w);
      y += widen<BF16>((uint16_t)(w >> 16));
    }
    sums[g * D + 2 * ch] = x;
    sums[g * D + 2 * ch + 1] = y;
  }
  __syncthreads();
  if constexpr (KG == 2) {
    // (behind the sums and the last tile's K, whose reads are over)
    float* const x = reinterpret_cast<float*>(lds + (lg ^ 1) * 4 * TB) + wave * (NDB * 8 + 1) * 64 + lane;
    for (int half = 0; half < 2; ++half) {               // half of the channel blocks at a time
      if (kg == 1) {
        if (half == 0) x[0] = dsum;
#pragma unroll
        for (int db = 0; db < NDB / 2; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[(1 + db * 16 + e) * 64] = half ? dq[NDB / 2 + db][e] : dq[db][e];
      }
      __syncthreads();
      if (kg == 0) {
        if (half == 0) dsum += x[0];
#pragma unroll
        for (int db = 0; db < NDB / 2; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (half) dq[NDB / 2 + db][e] += x[(1 + db * 16 + e) * 64];
            else dq[db][e] += x[(1 + db * 16 + e) * 64];
          }
      }
      __syncthreads();
    }
    if (kg == 1) return;
  }
  if (qi >= a.N) return;
  dsum += __shfl_xor(dsum, 32, 64);
  dsum *= 1.0f / (float)imax(1, imin(n - kl, BT));
  const float sq = a.rsd / f;
  uint16_t* o = (uint16_t*)a.dq + (((size_t)b * a.Hq + h) * a.N + qi) * D;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v4f c = v4f{};
      if (tl.count > 0)
#pragma unroll
        for (int g = 0; g < NG; ++g) c += *reinterpret_cast<const v4f*>(sums + g * D + 32 * db + 8 * q + 4 * hi);
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (dq[db][4 * q + e] - dsum * c[e]) * sq;
      *reinterpret_cast<v2u*>(o + 32 * db + 8 * q + 4 * hi) = qi < n ? v2u{pack16<BF16>(x[0], x[1]), pack16<BF16>(x[2], x[3])} : v2u{0u, 0u};
    }
}

// Chunks of the sinks' queries: enough workgroups for two per CU, at least 4 query
// tiles each.
int window_bwd_chunks(int B, int Hq, int Hkv, int N, int sinks) {
  const long long blocks = (long long)B * Hkv * cdiv(sinks, 32), tiles = (long long)cdiv(N, BT) * (Hq / Hkv);
  const long long want = 512 / (blocks > 0 ? blocks : 1), most = (tiles + 3) / 4;
  return (int)imax(1, (int)(want < most ? want : most));
}
// Query tiles per chunk of the other keys' dK and dV: one chunk where the longest block
// takes no more than 5/4 of what each of 512 workgroups (two per CU) would of the
// whole; else half of that whole's share, and 8 tiles at least (a chunk's part costs the
// traffic of about one).  2 x 12 / 4 heads of 1000 tokens, D = 64: 91 us in one chunk,
// 30 + 5 in up to 6 (join_keys_kernel is the 5).
int window_bwd_share(int B, int Hq, int Hkv, int N, int window, int* chunks) {
  long long total = 0;
  int most = 1;
  for (int k0 = 0; k0 < N; k0 += 128) {
    const TileRange r = query_tiles(k0, 128, N, N, window, false);
    total += r.t1 - r.t0;
    most = imax(most, r.t1 - r.t0);
  }
  const long long G = Hq / Hkv, each = (total * G * B * Hkv + 511) / 512;
  long long share = most * G;
  if (most * G * 4 > each * 5) share = each / 2 > 8 ? each / 2 : 8;
  *chunks = (int)((most * G + share - 1) / share);
  return (int)share;
}
size_t window_bwd_mpart_floats(int B, int Hkv, int N, int D, int chunks) {
  return chunks > 1 ? (size_t)B * Hkv * cdiv(N, 128) * chunks * 2 * 128 * D : 0;
}
size_t window_bwd_row_floats(int B, int Hq, int N) { return (size_t)B * Hq * ((N + BT - 1) / BT * BT); }
size_t window_bwd_norm_floats(int B, int Hq, int Hkv, int N) { return (size_t)B * (Hq + Hkv) * cdiv(N, PR); }
size_t window_bwd_part_floats(int B, int Hq, int Hkv, int N, int D, int sinks) {
  return (size_t)B * Hkv * cdiv(sinks, 32) * window_bwd_chunks(B, Hq, Hkv, N, sinks) * 2 * 32 * D;
}

template <int D, bool BF16>
static hipError_t launch_window_bwd_t(const WindowBwd& a, hipStream_t st) {
  hipLaunchKernelGGL((rows_kernel<D, BF16>), dim3((unsigned)cdiv(a.N, PR), (unsigned)(a.B * (a.Hq + (BF16 ? 0 : a.Hkv)))), dim3(256), 0,
                     st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!BF16) {
    hipLaunchKernelGGL(scale_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(64 * SW), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  // dQ first, as it may put delta right.  As in the forward: two groups of waves where
  // there is a workgroup per CU or less.
  const unsigned blocks = (unsigned)(a.B * a.Hq) * cdiv(a.N, 128);
  if (blocks <= 256) hipLaunchKernelGGL((dq_kernel<D, BF16, 2>), dim3(blocks), dim3(512), 0, st, a);
  else hipLaunchKernelGGL((dq_kernel<D, BF16, 1>), dim3(blocks), dim3(256), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const unsigned heads = (unsigned)(a.B * a.Hkv);
  hipLaunchKernelGGL((dkv_kernel<D, BF16, false>), dim3(heads * cdiv(a.N, 128) * a.mchunks), dim3(256), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.mchunks > 1) {
    hipLaunchKernelGGL((join_keys_kernel<D, BF16>), dim3((unsigned)cdiv(a.N, 512 / D), heads), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.sinks > 0) {
    hipLaunchKernelGGL((dkv_kernel<D, BF16, true>), dim3(heads * cdiv(a.sinks, 32) * a.chunks), dim3(128), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((join_sinks_kernel<D, BF16>), dim3((unsigned)a.sinks, heads), dim3(2 * D), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_window_bwd(const WindowBwd& a, int D, bool bf16, hipStream_t st) {
  if (D == 128) return bf16 ? launch_window_bwd_t<128, true>(a, st) : launch_window_bwd_t<128, false>(a, st);
  return bf16 ? launch_window_bwd_t<64, true>(a, st) : launch_window_bwd_t<64, false>(a, st);
}

}  // namespace sage
