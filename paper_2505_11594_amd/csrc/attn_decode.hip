// Attention of one new token per sequence over a paged cache, for gfx950.  The
// token is the last one of its sequence (length n, itself cached already); it
// sees key j iff j >= n - window or j < sinks.  Per key head and up to 16 query
// heads of its group:
//   S^T (keys x heads) = K . q^T,  online softmax in fp32,  O^T += V^T . P^T
// on v_mfma_f32_16x16x32: each cached row is read once for all heads of the
// group, 2 operations per byte and head, so the cache's bytes bound it and the
// unused columns of a small group cost nothing.  (131072 cached tokens, 32 / 8 heads: 16-bit
// 96-102 us, 5.3-5.6 TB/s; INT8 62-63 us, 4.4 TB/s: there the VALU, which widens the codes, is
// busy 54-59% of the time, and two waves per SIMD do not put all of it under the loads.)
//
// Every wave walks its own 32-key tiles: K goes from memory straight into the
// A operand's registers (lane l: key l % 16, channels 8 (l / 16) on), V through
// a wave-private LDS tile that is transposed as it is read; there is no barrier in
// the loop.  The next tile's rows are in flight while one is computed.
//
// The split: the visible tiles of all sequences, in steps of 4 tiles (one per
// wave), form one line that the workgroups of a key head cut into equal shares.
// A workgroup's share may span several short sequences, and a long sequence
// several workgroups: it is balanced whatever the lengths are, which only the
// device knows.  A part that is a whole sequence is final; others leave their
// (maximum, sum, O) for join_kernel.  A share has at most two of them: one that
// began before it (slot 0) and one that goes on behind it (slot 1).
//
// Infinities and NaN in values that the token sees: P enters its product in two parts, of
// which the second may be 0 or negative, and an infinity times it would be NaN.  But a
// channel's sums hold that channel's values only, and all heads see the same keys.  So a
// wave that would store anything but finite numbers looks through the part's rows of V once
// more for such values, and gives their channels what a sum with them is: an infinity, or
// NaN.  (A look at the sums per sequence for everyone else.  The same look before the waves'
// join took 14 registers of the tile loop.)
#include "lm_args.h"
#include "mma16.h"
#include "window.h"

namespace sage {

constexpr int DT = 32;                  // keys per tile
constexpr int DW = 4;                   // waves per workgroup
constexpr int DG = 16;                  // query heads per workgroup

__device__ __forceinline__ float max_over_groups(float x) {      // over the lanes l % 16 equal
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = smax(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return smax(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Steps of a sequence.
__device__ __forceinline__ TileList seq_tiles(const Decode& a, int s, int* n) {
  *n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size);
  return decode_tiles(*n, a.window, a.sinks, DT);
}

// The line of all sequences' steps.  Up to 64 sequences each wave adds up their steps
// itself, one per lane; of more, line_kernel has left the steps before each in
// a.before.
constexpr int LINE = 64;
struct Line {
  long long total, share;               // steps in all, and per workgroup
};
__device__ __forceinline__ int steps_of_lane(const Decode& a) {
  const int lane = threadIdx.x & 63;
  int n;
  return lane < a.c.S ? cdiv(seq_tiles(a, lane, &n).count, DW) : 0;
}
__device__ __forceinline__ int lanes_up_to(int x) {      // inclusive sum over the lanes
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}
__device__ __forceinline__ Line steps_line(const Decode& a, int sum) {
  Line l;
  l.total = a.before ? a.before[a.c.S] : __shfl(sum, 63, 64);
  l.share = (l.total + a.nw - 1) / a.nw;
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
__global__ __launch_bounds__(1024) void line_kernel(const Decode a) {
  __shared__ int red[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long long base = 0;
  for (int s0 = 0; s0 < a.c.S; s0 += 1024) {
    int n, c = 0;
    if (s0 + tid < a.c.S) c = cdiv(seq_tiles(a, s0 + tid, &n).count, DW);
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

// 16 int8 codes as 16 values of the type (exact).
template <bool BF16>
__device__ __forceinline__ void widen16(const v4i c, v4i& lo, v4i& hi) {
  uint32_t w[8];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int x = c[d];
    w[2 * d] = pack16<BF16>((float)(int8_t)x, (float)(int8_t)(x >> 8));
    w[2 * d + 1] = pack16<BF16>((float)(int8_t)(x >> 16), (float)(x >> 24));
  }
  lo = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
  hi = v4i{(int)w[4], (int)w[5], (int)w[6], (int)w[7]};
}

// Of 8 values, bit e of pos: value e is +infinity or NaN, of neg: -infinity or NaN.
template <bool BF16>
__device__ __forceinline__ void find_nonfinite(const v4i x, unsigned& pos, unsigned& neg) {
  constexpr uint32_t INF = BF16 ? 0x7F80u : 0x7C00u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t h = (uint32_t)x[e / 2] >> (16 * (e & 1)) & 0xFFFFu, size = h & 0x7FFFu;
    if (size > INF || h == INF) pos |= 1u << e;
    if (size > INF || h == (INF | 0x8000u)) neg |= 1u << e;
  }
}

// BF16: the type of q and o.  I8: 8-bit cache; its codes are exact in either type,
// and P times V's scale, whose size nothing bounds, is taken in bf16.  P enters its
// product with V in two parts, rounded and rest (together 2^-16 of it in bf16, 2^-22 in
// fp16): the matrix instructions have the time.  (D = 64 is held to the 168 registers that
// let three waves on a SIMD; left alone it takes 171.)
template <int D, bool BF16, bool I8>
__global__ __launch_bounds__(64 * DW, D == 64 ? 3 : 2) void paged_decode_kernel(const Decode a) {
  constexpr bool PB = BF16 || I8;                        // type of P and V in the second product
  constexpr int EB = I8 ? 1 : 2, ROW = D * 2;
  constexpr int KL = D * EB / 64;                        // 16-byte K loads per lane and 16-key subtile
  constexpr int RC = D * EB / 16, VR = 64 / RC, VL = DT / VR;   // V: chunks per row, rows per load, loads
  constexpr int NKS = D / 32, NDB = D / 16;
  constexpr int PADQ = D + 4;                            // floats per head in the waves' join
  constexpr int REG = DG * PADQ * 4;                     // LDS bytes per wave: V tile, then its O
  static_assert(REG >= DT * ROW && REG % 256 == 0, "a V tile fits; addresses inside it are xor-ed");
  __shared__ __attribute__((aligned(256))) uint8_t lds[DW * REG + DW * DG * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, grp = lane >> 4;
  const int hk = blockIdx.y, G = a.Hq / a.c.Hkv, g0 = blockIdx.z * DG, gn = min(DG, G - g0);
  const int h0 = hk * G + g0;                            // first query head
  uint8_t* const vt = lds + wave * REG;
  const uint32_t vbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)vt;
  // block db's transposing read: vat ^ 32 db (rows start on multiples of their size)
  const uint32_t vat = vbase + (4 * grp + c16 / 4) * ROW + vswz<D>(4 * grp + c16 / 4, (c16 & 3) / 2) * 16 + 8 * (c16 & 1);

  long long r0 = 0, r1 = 0, before = 0;
  int s = blockIdx.x, mine = 0, upto = 0;
  if (a.nw > 0) {
    if (!a.before) {
      mine = steps_of_lane(a);
      upto = lanes_up_to(mine);
    }
    const Line line = steps_line(a, upto);
    r0 = min(line.total, blockIdx.x * line.share);
    r1 = min(line.total, r0 + line.share);
    if (r0 >= r1) return;
    s = find_step(a, mine, upto, r0, &before);
  }
  const int ps = a.c.page_size;
  for (;;) {
    // one sequence (or the share's part of it)
    s = __builtin_amdgcn_readfirstlane(s);
    int n;
    const TileList tl = seq_tiles(a, s, &n);
    const int steps = cdiv(tl.count, DW);
    const int off = a.nw > 0 ? (int)(r0 - before) : 0;
    const int cnt = a.nw > 0 ? (int)min((long long)(steps - off), r1 - r0) : steps;
    const int tend = min(tl.count, DW * (off + cnt));
    const int32_t* const table = a.c.table + (size_t)s * a.c.max_pages;

    v4i qreg[NKS];
    {
      const uint16_t* q = (const uint16_t*)a.q + s * a.q_s + (h0 + min(c16, gn - 1)) * a.q_h;
#pragma unroll
      for (int i = 0; i < NKS; ++i)                      // channels in the order in which K's lie in its registers
        qreg[i] = *reinterpret_cast<const v4i*>(q + (I8 ? 64 * (i / 2) + 16 * grp + 8 * (i & 1) : 32 * i + 8 * grp));
    }
    v4f oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = v4f{};
    float m = -INFINITY, l = 0.0f;                       // m in log2 units

    // the page of this lane's key (key l % 32 of a tile), -1 where it has none
    auto page_of = [&](int i) -> int {
      const int key = tl.tile(i) * DT + (lane & 31);
      if (i >= tend || !decode_sees(key, n, a.window, a.sinks)) return -1;
      const int id = table[key / ps];
      return page_ok(id, a.c.pages) ? id : -1;
    };
    struct Rows {
      v4i k[2][KL], v[VL];
      float ks[2], vs;
    };
    auto load = [&](int i, int id, Rows& r) {
      const int kb = tl.tile(i) * DT;
      const int slot = max(id, 0) == id ? (kb + (lane & 31)) % ps : 0;      // rows without a page: the cache's first one
      const int pid = max(id, 0);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int p = __shfl(pid, 16 * t + c16, 64), sl = __shfl(slot, 16 * t + c16, 64);
        const uint8_t* k = (const uint8_t*)a.c.k + EB * (p * a.c.ks.b + hk * a.c.ks.h + sl * a.c.ks.n);
#pragma unroll
        for (int j = 0; j < KL; ++j) r.k[t][j] = *reinterpret_cast<const v4i*>(k + 64 * j + 16 * grp);
      }
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int row = VR * j + lane / RC;
        const int p = __shfl(pid, row, 64), sl = __shfl(slot, row, 64);
        const uint8_t* v = (const uint8_t*)a.c.v + EB * (p * a.c.vs.b + hk * a.c.vs.h + sl * a.c.vs.n);
        r.v[j] = *reinterpret_cast<const v4i*>(v + 16 * (lane % RC));
      }
      if constexpr (I8) {
        const size_t x = ((size_t)pid * a.c.Hkv + hk) * ps + slot;
        r.ks[0] = a.c.k_scale[x];
        r.vs = id >= 0 ? a.c.v_scale[x] : 0.0f;          // a key that is not seen adds nothing, whatever lies there
      }
    };

    int i = DW * off + wave;
    int id = page_of(i), id1 = page_of(i + DW);
    Rows cur, nxt;
    if (i < tend) load(i, id, cur);
    for (; i < tend; i += DW) {
      const int id2 = page_of(i + 2 * DW);
      if (i + DW < tend) load(i + DW, id1, nxt);
      const unsigned ok = (unsigned)__builtin_amdgcn_ballot_w64(id >= 0);    // bit: key of the tile (both halves alike)

      // scores of keys 16 t + 4 grp + e
      v4f sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        v4f acc = v4f{};
        if constexpr (I8) {
#pragma unroll
          for (int j = 0; j < KL; ++j) {
            v4i lo, hi;
            widen16<BF16>(cur.k[t][j], lo, hi);
            acc = mma16<BF16>(lo, qreg[2 * j], acc);
            acc = mma16<BF16>(hi, qreg[2 * j + 1], acc);
          }
        } else {
#pragma unroll
          for (int j = 0; j < KL; ++j) acc = mma16<BF16>(cur.k[t][j], qreg[j], acc);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = acc[e] * a.c2;
          const int key = 16 * t + 4 * grp + e;
          if constexpr (I8) x *= __shfl(cur.ks[0], key, 64);
          sc[t][e] = (ok >> key) & 1u ? x : -INFINITY;
        }
      }
      if (a.scores && c16 < gn) {
        float* row = a.scores + ((size_t)s * a.Hq + h0 + c16) * a.score_stride + tl.tile(i) * DT;
        *reinterpret_cast<v4f*>(row + 4 * grp) = sc[0];
        *reinterpret_cast<v4f*>(row + 16 + 4 * grp) = sc[1];
      }
      float x = sc[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) x = smax(x, sc[e >> 2][e & 3]);
      const float m_new = smax(m, max_over_groups(x));
      const float mc = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - mc);
      m = m_new;
      const float mp = mc - kPShift<PB>;
      float sum = 0.0f;
      v4i pk, pl;                                        // P's upper part, and what its rounding left
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float p0 = __builtin_amdgcn_exp2f(sc[e >> 2][e & 3] - mp), p1 = __builtin_amdgcn_exp2f(sc[e >> 2][(e & 3) + 1] - mp);
        sum += p0 + p1;
        if constexpr (I8) {
          const int key = 16 * (e >> 2) + 4 * grp + (e & 3);
          p0 *= __shfl(cur.vs, key, 64);
          p1 *= __shfl(cur.vs, key + 1, 64);
        }
        const uint32_t hw = pack16<PB>(p0, p1);
        pk[e / 2] = (int)hw;
        pl[e / 2] = (int)pack16<PB>(p0 - widen<PB>((uint16_t)hw), p1 - widen<PB>((uint16_t)(hw >> 16)));
      }
      l = l * alpha + sum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[db][e] *= alpha;
      }
      // V into the wave's tile; rows that are not seen are zero, whatever lies in the cache
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int row = VR * j + lane / RC, ch = lane % RC;
        v4i v = cur.v[j];
        if (!((ok >> row) & 1u)) v = v4i{};
        if constexpr (I8) {
          v4i lo, hi;
          widen16<true>(v, lo, hi);
          *reinterpret_cast<v4i*>(vt + row * ROW + vswz<D>(row, 2 * ch) * 16) = lo;
          *reinterpret_cast<v4i*>(vt + row * ROW + vswz<D>(row, 2 * ch + 1) * 16) = hi;
        } else {
          *reinterpret_cast<v4i*>(vt + row * ROW + vswz<D>(row, ch) * 16) = v;
        }
      }
      const uint32_t va = opaque(vat);
      static_for<NDB / 4>([&](auto B_) {
        constexpr int b4 = 4 * decltype(B_)::value;
        v8bf vv[4];                                      // 32 keys of 4 channel blocks: two reads each, 16 keys apart
        vt_read4<0, 16 * ROW>(va ^ (32 * b4), va ^ (32 * b4 + 32), va ^ (32 * b4 + 64), va ^ (32 * b4 + 96), vv[0], vv[1], vv[2], vv[3]);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const v4i x = __builtin_bit_cast(v4i, vv[d]);
          oacc[b4 + d] = mma16<PB>(x, pl, mma16<PB>(x, pk, oacc[b4 + d]));
        }
      });
      id = id1;
      id1 = id2;
      cur = nxt;
    }

    // join the 4 waves
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    float* const ml = reinterpret_cast<float*>(lds + DW * REG);
    if (grp == 0) {
      ml[(wave * DG + c16) * 2] = m;
      ml[(wave * DG + c16) * 2 + 1] = l;
    }
    __syncthreads();                                     // also: every wave is past its last V tile
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < DW; ++w) mm = smax(mm, ml[(w * DG + c16) * 2]);
    const float mc = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < DW; ++w) ll += ml[(w * DG + c16) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * DG + c16) * 2] - mc);
    const float f = __builtin_amdgcn_exp2f(m - mc);
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      *reinterpret_cast<v4f*>(vt + (c16 * PADQ + 16 * db + 4 * grp) * 4) = oacc[db] * v4f{f, f, f, f};
    __syncthreads();

    const bool whole = off == 0 && cnt == steps;
    const size_t slot = (size_t)blockIdx.x * 2 + (off == 0 ? 1 : 0);
    if (wave == 0 && grp == 0 && c16 < gn) {
      const float l2 = ll > 0.0f || ll != ll ? mm + (__builtin_log2f(ll) - kPShift<PB>) : -INFINITY;
      if (whole) {
        if (a.lse) a.lse[(size_t)s * a.Hq + h0 + c16] = l2 * 0.69314718055994530942f;
        if (a.lse2) a.lse2[(size_t)s * a.Hq + h0 + c16] = l2;
      } else {
        float* p = a.part + (size_t)a.nw * 2 * a.Hq * D + (slot * a.Hq + h0 + c16) * 2;
        p[0] = mm;
        p[1] = ll;
      }
    }
    // thread: head tid / 16, 4 channels at a time
    const int qh = tid >> 4;
    const float lq = __shfl(ll, qh, 64);                 // lane qh (< 16) holds head qh's sum
    v4f x[D / 64];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      x[c] = v4f{};
#pragma unroll
      for (int w = 0; w < DW; ++w) x[c] += *reinterpret_cast<const v4f*>(lds + w * REG + (qh * PADQ + 64 * c + 4 * (tid & 15)) * 4);
    }
    if constexpr (!I8) {
      bool odd = false;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= !(__builtin_fabsf(x[c][e]) < INFINITY);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        unsigned pos = 0, neg = 0;                       // of channels 8 (lane % RC) + e
#pragma unroll 1
        for (int t = DW * off; t < tend; ++t) {
          const int id = page_of(t), at = (tl.tile(t) * DT + (lane & 31)) % ps;
#pragma unroll 1
          for (int j = 0; j < VL; ++j) {
            const int row = VR * j + lane / RC, p = __shfl(id, row, 64), sl = __shfl(at, row, 64);
            const uint8_t* v = (const uint8_t*)a.c.v + EB * (max(p, 0) * a.c.vs.b + hk * a.c.vs.h + sl * a.c.vs.n) + 16 * (lane % RC);
            if (p >= 0) find_nonfinite<BF16>(*reinterpret_cast<const v4i*>(v), pos, neg);
          }
        }
#pragma unroll
        for (int o = RC; o < 64; o <<= 1) {              // over the rows
          pos |= __shfl_xor(pos, o, 64);
          neg |= __shfl_xor(neg, o, 64);
        }
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {               // channel 64 c + 4 (tid % 16) + e
          const int from = 8 * c + (lane & 15) / 2, bit = 4 * (lane & 1);
          const unsigned p = __shfl(pos, from, 64) >> bit, n = __shfl(neg, from, 64) >> bit;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((p | n) >> e & 1u) x[c][e] = (p >> e & 1u ? INFINITY : 0.0f) - (n >> e & 1u ? INFINITY : 0.0f);
        }
      }
    }
    if (qh < gn) {
      const float inv = lq > 0.0f || lq != lq ? 1.0f / lq : 0.0f;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const int d = 64 * c + 4 * (tid & 15);
        if (whole) {
          const v2u o = {pack16<BF16>(x[c][0] * inv, x[c][1] * inv), pack16<BF16>(x[c][2] * inv, x[c][3] * inv)};
          *reinterpret_cast<v2u*>((uint16_t*)a.o + ((size_t)s * a.Hq + h0 + qh) * D + d) = o;
        } else {
          *reinterpret_cast<v4f*>(a.part + (slot * a.Hq + h0 + qh) * D + d) = x[c];
        }
      }
    }
    if (a.nw == 0) return;
    r0 += cnt;
    if (r0 >= r1) return;
    s = find_step(a, mine, upto, r0, &before);           // the next one that has steps
    __syncthreads();                                     // the next sequence's V tiles overwrite the join's LDS
  }
}

// Sequences whose steps several workgroups shared: O = sum O_w 2^(m_w - m) / l.
// One workgroup per (sequence, query head); its waves take every fourth part.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_kernel(const Decode a, float shift) {
  constexpr int CL = D / 64;                             // channels per lane
  __shared__ float sums[4][D + 1];
  const int s = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mine = a.before ? 0 : steps_of_lane(a), upto = a.before ? 0 : lanes_up_to(mine);
  const Line line = steps_line(a, upto);
  const long long before = a.before ? a.before[s] : __shfl(upto - mine, s, 64);
  const int steps = a.before ? (int)(a.before[s + 1] - before) : __shfl(mine, s, 64);
  const int w0 = steps > 0 ? (int)(before / line.share) : 0, w1 = steps > 0 ? (int)((before + steps - 1) / line.share) : -1;
  if (w0 == w1) return;                                  // final already
  const float* ml = a.part + (size_t)a.nw * 2 * a.Hq * D;
  // a share's slot 1 if the sequence begins in it, slot 0 if it began before
  auto at = [&](int w) { return ((size_t)w * 2 + (w == w0 ? 1 : 0)) * a.Hq + h; };
  float m = -INFINITY, l = 0.0f, x[CL] = {};
  for (int w = w0 + lane; w <= w1; w += 64) m = smax(m, ml[at(w) * 2]);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = smax(m, __shfl_xor(m, d, 64));
  const float mc = m == -INFINITY ? 0.0f : m;
#pragma unroll 8
  for (int w = w0 + wave; w <= w1; w += 4) {
    const float f = __builtin_amdgcn_exp2f(ml[at(w) * 2] - mc);
    l += ml[at(w) * 2 + 1] * f;
    const float* p = a.part + at(w) * D + lane * CL;
#pragma unroll
    for (int i = 0; i < CL; ++i) x[i] += __builtin_fabsf(p[i]) < INFINITY ? p[i] * f : p[i];   // (an infinity stays one where f is 0)
  }
#pragma unroll
  for (int i = 0; i < CL; ++i) sums[wave][lane * CL + i] = x[i];
  if (lane == 0) sums[wave][D] = l;
  __syncthreads();
  if (wave > 0) return;
  l = (sums[0][D] + sums[1][D]) + (sums[2][D] + sums[3][D]);
  const float l2 = l > 0.0f || l != l ? m + (__builtin_log2f(l) - shift) : -INFINITY;
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
  for (int i = 0; i < CL; ++i) {
    const int c = lane * CL + i;
    x[i] = ((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c])) * inv;
  }
  uint16_t* o = (uint16_t*)a.o + ((size_t)s * a.Hq + h) * D + lane * CL;
  if constexpr (D == 128) *reinterpret_cast<uint32_t*>(o) = pack16<BF16>(x[0], x[1]);
  else *o = (uint16_t)pack16<BF16>(x[0], 0.0f);
  if (lane == 0) {
    if (a.lse) a.lse[(size_t)s * a.Hq + h] = l2 * 0.69314718055994530942f;
    if (a.lse2) a.lse2[(size_t)s * a.Hq + h] = l2;
  }
}

// weights[j] += sum over the group's heads of exp(S - L), four cached tokens per thread.
// Bound by the scores' bytes, if enough of them are on their way: 48 sequences of up to
// 8000 tokens, 32 heads (34 MB in all) take 10 us, 18 with a wait for each head's.
__global__ __launch_bounds__(256) void add_weights_kernel(const Decode a) {
  const int s = blockIdx.z, hk = blockIdx.y, G = a.Hq / a.c.Hkv;
  const int n = cached_len(a.lens[s], a.c.max_pages * a.c.page_size);
  float* w = a.weights + ((size_t)s * a.c.Hkv + hk) * a.wstride;
  const float* sc = a.scores + ((size_t)s * a.Hq + (size_t)hk * G) * a.score_stride;
  const float* l2 = a.lse2 + (size_t)s * a.Hq + hk * G;
  for (int j = (blockIdx.x * 256 + threadIdx.x) * 4; j < n; j += gridDim.x * 1024) {
    // (the scores of a tile of 32 are written together, those of unseen keys as -inf; other tiles hold nothing)
    bool see[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) see[e] = decode_sees(j + e, n, a.window, a.sinks);
    if (!(see[0] || see[1] || see[2] || see[3])) continue;
    float old[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) old[e] = w[imin(j + e, n - 1)];   // (no branches between the loads)
    v4f x = v4f{};
    for (int g0 = 0; g0 < G; g0 += 4) {                  // loads of several heads in flight, behind no branch
      v4f y[4];
      float l[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int g = imin(g0 + u, G - 1);
        y[u] = *reinterpret_cast<const v4f*>(sc + g * a.score_stride + j);
        l[u] = l2[g];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(y[u][e] - l[u]);
          x[e] += g0 + u < G && y[u][e] != -INFINITY ? p : 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (see[e]) w[j + e] = old[e] + x[e];
  }
}

// Workgroups per group of 16 query heads of a key head.  Two fit a CU, so 512 in
// all keep every CU busy; a batch has no use for more than its steps.  Sequences of
// up to 4 steps (512 cached tokens) get a workgroup each instead, and no join.
int decode_workgroups(int S, int Hq, int Hkv, int capacity) {
  const long long steps = cdiv(capacity, DT * DW) + 1;   // the sinks' tiles may add a step
  if (steps <= 5) return 0;
  const int heads = Hkv * cdiv(Hq / Hkv, DG);
  const long long want = imax(1, 512 / heads), most = (long long)S * steps;
  return (int)(want < most ? want : most);
}
size_t decode_part_floats(int S, int Hq, int Hkv, int D, int capacity) {
  return (size_t)decode_workgroups(S, Hq, Hkv, capacity) * 2 * Hq * (D + 2);
}

size_t decode_line_longs(int S, int Hq, int Hkv, int capacity) {
  return S > LINE && decode_workgroups(S, Hq, Hkv, capacity) > 0 ? (size_t)S + 1 : 0;
}

template <int D, bool BF16>
static hipError_t launch_decode_t(const Decode& a, hipStream_t st) {
  const int G = a.Hq / a.c.Hkv;
  const dim3 grid((unsigned)(a.nw > 0 ? a.nw : a.c.S), (unsigned)a.c.Hkv, (unsigned)cdiv(G, DG)), block(64 * DW);
  hipError_t e = hipSuccess;
  if (a.before) {
    hipLaunchKernelGGL(line_kernel, dim3(1), dim3(1024), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.c.k_scale) hipLaunchKernelGGL((paged_decode_kernel<D, BF16, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_decode_kernel<D, BF16, false>), grid, block, 0, st, a);
  e = hipGetLastError();
  if (e == hipSuccess && a.nw > 0) {
    const float shift = a.c.k_scale ? 0.0f : kPShift<BF16>;
    hipLaunchKernelGGL((join_kernel<D, BF16>), dim3((unsigned)a.c.S, (unsigned)a.Hq), dim3(256), 0, st, a, shift);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.weights) {
    const int capacity = a.c.max_pages * a.c.page_size;
    const int want = imax(1, (int)(2048 / ((long long)a.c.S * a.c.Hkv)));
    hipLaunchKernelGGL(add_weights_kernel, dim3((unsigned)imin(cdiv(capacity, 1024), want), (unsigned)a.c.Hkv, (unsigned)a.c.S),
                       dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_paged_decode(const Decode& a, int D, bool bf16, hipStream_t st) {
  if (D == 128) return bf16 ? launch_decode_t<128, true>(a, st) : launch_decode_t<128, false>(a, st);
  return bf16 ? launch_decode_t<64, true>(a, st) : launch_decode_t<64, false>(a, st);
}

}  // namespace sage
