// Attention of one new token per sequence over a paged cache in MXFP4 (E2M1 codes, an
// E8M0 scale per 32 channels of a token and head), for gfx950.  The mathematics, the walk
// and the split are those of attn_decode.hip; what differs is how 4 bits reach the matrix
// instructions.
//
// The codes are widened to bf16 with their scales, two values an instruction and exactly, and
// both products run on v_mfma_f32_16x16x32_bf16: K's codes go from memory straight into the A
// operand's registers; V's into a wave-private LDS tile that is transposed as it is read.  q of
// fp16 enters in two bf16 parts (exact), P in two for either type.
// (The block-scaled product takes K as it lies in memory, times q in E4M3 parts; its sums of
// parts that differ in size are off by 2^-18 of their terms, so L was by 8e-5.)
//
// (131072 tokens, 32 / 8 heads: the kernel takes 29-30 us, 4.8 TB/s, and 5 for the join: HBM, after 4 us
// before the first and behind the last tile.  VALU busy 38% of the time, LDS 35%, MFMAs 20%.)
//
// A group of up to 4 (8) query heads leaves 12 (8) of the product's 16 columns free: its
// heads stand there 4 (2) times, and each copy takes the softmax of another 16 (32) of
// the tile's 64 keys.  P is brought together again within the rows of 16 lanes.
#include "decode_split.h"

namespace sage {

namespace {

constexpr int FT = 64;                  // keys per tile
constexpr int FW = 4;                   // waves per workgroup

// 8 values of q in bf16: rounded, and of fp16 what the rounding left (11 bits in 8 and 8: exact).
template <bool BF16>
__device__ __forceinline__ void split_q(const v4i v, v4i* hi, v4i* lo) {
  if constexpr (BF16) {
    *hi = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x0 = fp16_to_f32((uint16_t)v[i]), x1 = fp16_to_f32((uint16_t)((uint32_t)v[i] >> 16));
      const uint32_t h = pack16<true>(x0, x1);
      (*hi)[i] = (int)h;
      (*lo)[i] = (int)pack16<true>(x0 - bf16_to_f32((uint16_t)h), x1 - bf16_to_f32((uint16_t)(h >> 16)));
    }
  }
}

// 8 codes as bf16 values times a power of two.
__device__ __forceinline__ v4i widen_fp4(int codes, float scale) {
  v4i r;
  r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes, scale, 0));
  r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes, scale, 1));
  r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes, scale, 2));
  r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes, scale, 3));
  return r;
}

template <int CTRL>
__device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true); }
constexpr int kLanesOn = 0x100, kTurn = 0x120;           // + n: lane i takes lane i + n (0 past the row of 16); rows turned by n

// The lowest x bits.
__device__ __forceinline__ unsigned long long low_bits(int x) { return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1; }

// A transposing read: 16 keys (rows) by 16 channels of the wave's V tile.
__device__ __forceinline__ v2u tr_read(uint32_t at) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)at));
}

// WHOLE: the 16 keys of a subtile lie on one page, K and V lie alike, and each has at most
// 2^31 bytes: a subtile's place is found once for the wave, in scalar registers.  (17 to 35 of what else is
// scalar lie in lanes of a vector register for it, read per sequence, not per tile.  Not only to save
// instructions: a launch does not find its code in the caches.  5 KB more of it, for two tiles'
// rows in flight, made every call 1 to 2.5 us longer.)
// SCORES: they are kept for the weights, which another launch adds up (32 sequences of 857 to 6000 tokens, 32 / 8
// heads, in a graph of calls: 43 us, 34 without: 14 MB written and read, and a launch).
template <int D, bool BF16, int COPIES, bool WHOLE, bool SCORES>
__global__ __launch_bounds__(64 * FW, 2) void paged_decode_fp4_kernel(const Decode a) {
  constexpr int ROW = D * 2, SB = D / 32;                // bytes of a V row in LDS; scale bytes of a cached row
  constexpr int HC = 16 / COPIES, TS = 4 / COPIES;       // heads per copy; subtiles of 16 keys whose softmax a copy takes
  constexpr int NKS = D / 32;                            // steps of 32 channels of S; lane: 8 channels of each, D / 4 in a row
  constexpr int NDB = D / 16;
  constexpr int PADQ = D + 4;
  constexpr int REG = D == 128 ? 33 * 256 : 17 * 256;    // LDS bytes per wave: 32 rows of V, then its O
  static_assert(REG >= DG * PADQ * 4 && REG >= 32 * ROW && REG % 256 == 0, "both fit; addresses inside a tile are xor-ed");
  __shared__ __attribute__((aligned(256))) uint8_t lds[FW * REG + FW * DG * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, grp = lane >> 4, copy = c16 / HC, head = c16 % HC;
  const int hk = blockIdx.y, G = a.Hq / a.c.Hkv, g0 = blockIdx.z * DG, gn = imin(DG, G - g0);
  const int h0 = hk * G + g0;                            // first query head
  uint8_t* const vt = lds + wave * REG;
  const uint32_t vbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)vt;
  const uint32_t vat = vbase + (4 * grp + c16 / 4) * ROW + vswz<D>(4 * grp + c16 / 4, (c16 & 3) / 2) * 16 + 8 * (c16 & 1);

  const uint32_t wat = vbase + c16 * ROW + vswz<D>(c16, NKS * grp) * 16;   // its row c16's chunk; the next ones by xor

  long long r0 = 0, r1 = 0, before = 0;
  int s = blockIdx.x, mine = 0, upto = 0, length = 0;    // mine, length: of sequence `lane`
  if (a.nw > 0) {
    if (!a.before) {
      mine = steps_of_lane<FT, FW>(a, &length);
      upto = lanes_up_to(mine);
    }
    const Line line = steps_line(a, upto);
    r0 = min(line.total, blockIdx.x * line.share);
    r1 = min(line.total, r0 + line.share);
    if (r0 >= r1) return;
    s = find_step(a, mine, upto, r0, &before);
  }
  const int ps = a.c.page_size;
  // this key head's rows and scales of page 0; a lane's bytes from its subtile's first row on:
  // key c16, channels from D / 4 grp on, and their scale
  const uint8_t* const k_rows = (const uint8_t*)a.c.k + hk * a.c.ks.h;
  const uint8_t* const v_rows = (const uint8_t*)a.c.v + hk * a.c.vs.h;
  const uint8_t* const k_scale = (const uint8_t*)a.c.k_scale + (size_t)hk * ps * SB;
  const uint8_t* const v_scale = (const uint8_t*)a.c.v_scale + (size_t)hk * ps * SB;
  const uint32_t row_at = (uint32_t)c16 * (uint32_t)a.c.ks.n + D / 8 * grp, scale_at = c16 * SB + D * grp / 128;
  const __amdgpu_buffer_rsrc_t k_buf = make_rsrc(k_rows, 0x80000000u), v_buf = make_rsrc(v_rows, 0x80000000u);
  const __amdgpu_buffer_rsrc_t ks_buf = make_rsrc(k_scale, 0x80000000u), vs_buf = make_rsrc(v_scale, 0x80000000u);
  // A sequence, or the share's part of it.
  struct Part {
    int s, n, off, cnt, steps, tend;
    TileList tl;
    const int32_t* table;
  };
  auto part_of = [&](int s, long long before) {
    Part g;
    g.s = __builtin_amdgcn_readfirstlane(s);
    g.n = __builtin_amdgcn_readfirstlane(a.nw > 0 && !a.before ? __shfl(length, g.s, 64) : cached_len(a.lens[g.s], a.c.max_pages * ps));
    g.tl = decode_tiles(g.n, a.window, a.sinks, FT);
    g.steps = cdiv(g.tl.count, FW);
    g.off = a.nw > 0 ? __builtin_amdgcn_readfirstlane((int)(r0 - before)) : 0;
    g.cnt = a.nw > 0 ? __builtin_amdgcn_readfirstlane((int)min((long long)(g.steps - g.off), r1 - r0)) : g.steps;
    g.tend = imin(g.tl.count, FW * (g.off + g.cnt));
    g.table = a.c.table + (size_t)g.s * a.c.max_pages;
    return g;
  };
  // Where a tile's keys lie.  WHOLE: its subtiles' pages (-1: none) and first slots; subtiles behind
  // the sequence's last key stand for the last one.  Else of this lane's key (key `lane` of the tile).
  struct Place {
    int page[WHOLE ? 4 : 1], slot[WHOLE ? 4 : 1];
  };
  auto place_of = [&](const Part& g, int i) {
    Place p;
    if constexpr (WHOLE) {
      const int kt = g.tl.tile(imin(i, g.tend - 1)) * FT, last = (g.n - 1) & ~15;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int kb = imax(0, imin(kt + 16 * t, last)), j = a.per_page(kb);
        p.page[t] = ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)g.table)[j];
        p.slot[t] = kb - j * ps;
      }
    } else {
      const int key = g.tl.tile(i) * FT + lane, j = a.per_page(key);
      p.page[0] = -1;
      p.slot[0] = key - j * ps;
      if (i < g.tend && decode_sees(key, g.n, a.window, a.sinks)) p.page[0] = g.table[j];
    }
    return p;
  };
  // Which keys of the tile are seen, one bit each.
  auto seen_of = [&](const Part& g, int i, const Place& p) {
    if constexpr (WHOLE) {
      const int kt = g.tl.tile(i) * FT;
      unsigned long long x = ~0ull;
      if (kt + FT > g.n || (kt < g.n - a.window && kt + FT > a.sinks))
        x = low_bits(g.n - kt) & (~low_bits(g.n - a.window - kt) | low_bits(a.sinks - kt));
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (!page_ok(p.page[t], a.c.pages)) x &= ~(0xFFFFull << (16 * t));
      return x;
    } else {
      return (unsigned long long)__builtin_amdgcn_ballot_w64(page_ok(p.page[0], a.c.pages));
    }
  };
  struct Rows {
    int x[4][NKS], scale[4];                             // key 16 t + c16, channels from D / 4 grp on
  };
  // The rows' bytes from the first one on (WHOLE); keys without a page get rows of the cache's first one.
  struct Offsets {
    uint32_t row[4], scale[4];
  };
  auto offsets_of = [&](const Place& p) {
    Offsets o;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t ok = page_ok(p.page[WHOLE ? t : 0], a.c.pages) ? ~0u : 0u;
      const uint32_t page = (uint32_t)p.page[WHOLE ? t : 0] & ok, slot = (uint32_t)p.slot[WHOLE ? t : 0] & ok;
      o.row[t] = page * (uint32_t)a.c.ks.b + slot * (uint32_t)a.c.ks.n;
      o.scale[t] = (page * (uint32_t)(a.c.Hkv * ps) + slot) * SB;
    }
    return o;
  };
  // Behind the last tile a load has no bytes (WHOLE): with a branch around it the compiler would count
  // on none being in flight behind those of the tile at work, and wait for all (131072 tokens: 46 -> 37 us).
  auto load = [&](const Part& g, int i, const Offsets& o, __amdgpu_buffer_rsrc_t rows, __amdgpu_buffer_rsrc_t scales, Rows& r) {
    const uint32_t none = i < g.tend ? 0u : 0x80000000u;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (D == 128)
        *reinterpret_cast<v4i*>(r.x[t]) = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rows, row_at | none, o.row[t], 0));
      else
        *reinterpret_cast<v2u*>(r.x[t]) = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(rows, row_at | none, o.row[t], 0));
      r.scale[t] = __builtin_amdgcn_raw_buffer_load_b8(scales, scale_at | none, o.scale[t], 0);
    }
  };
  auto load_each = [&](const Part& g, int i, const Place& pl, const uint8_t* rows, const Strides& st, const uint8_t* scales, Rows& r) {
    if (i >= g.tend) return;
    const bool ok = page_ok(pl.page[0], a.c.pages);
    const int pid = ok ? pl.page[0] : 0, place = ok ? pl.slot[0] : 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int page = __shfl(pid, 16 * t + c16, 64), slot = __shfl(place, 16 * t + c16, 64);
      const uint8_t* p = rows + (page * st.b + slot * st.n) + D / 8 * grp;
      if constexpr (D == 128) *reinterpret_cast<v4i*>(r.x[t]) = *reinterpret_cast<const v4i*>(p);
      else *reinterpret_cast<v2u*>(r.x[t]) = *reinterpret_cast<const v2u*>(p);
      r.scale[t] = scales[((size_t)page * a.c.Hkv * ps + slot) * SB + D * grp / 128];
    }
  };
  for (;;) {
    const Part now = part_of(s, before);
    const int tend = now.tend;
    // K's registers are filled again when the scores have used them, V's when it lies in LDS.
    int i = FW * now.off + wave;
    Place at = place_of(now, i), at1 = place_of(now, i + FW);
    Rows kr, vr;
    if constexpr (WHOLE) {
      const Offsets o = offsets_of(at);
      load(now, i, o, k_buf, ks_buf, kr);
      load(now, i, o, v_buf, vs_buf, vr);
    } else {
      load_each(now, i, at, k_rows, a.c.ks, k_scale, kr);
      load_each(now, i, at, v_rows, a.c.vs, v_scale, vr);
    }
    v4i qreg[NKS], qrest[BF16 ? 1 : NKS];                // channels in the order in which K's lie in its registers
    {
      const uint16_t* q = (const uint16_t*)a.q + now.s * a.q_s + (h0 + imin(head, gn - 1)) * a.q_h + D / 4 * grp;
#pragma unroll
      for (int j = 0; j < NKS; ++j) split_q<BF16>(*reinterpret_cast<const v4i*>(q + 8 * j), &qreg[j], &qrest[BF16 ? 0 : j]);
    }
    v4f oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = v4f{};
    float m = -INFINITY, l = 0.0f;                       // m in log2 units
    for (; i < tend; i += FW) {
      const Place at2 = place_of(now, i + 2 * FW);
      const unsigned long long ok = seen_of(now, i, at);

      // scores of keys 16 t + 4 grp + e, of which this lane takes t = TS copy + u
      v4f acc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] = v4f{};
#pragma unroll
      for (int j = 0; j < NKS; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const v4i k = widen_fp4(kr.x[t][j], __uint_as_float((uint32_t)kr.scale[t] << 23));
          if constexpr (!BF16) acc[t] = mma16<true>(k, qrest[j], acc[t]);
          acc[t] = mma16<true>(k, qreg[j], acc[t]);
        }
      __builtin_amdgcn_sched_barrier(0);                 // (phases kept apart: the registers of one serve the next)
      Offsets o;
      if constexpr (WHOLE) {
        o = offsets_of(at1);
        load(now, i + FW, o, k_buf, ks_buf, kr);
      } else {
        load_each(now, i + FW, at1, k_rows, a.c.ks, k_scale, kr);
      }
      float sc[TS][4];
#pragma unroll
      for (int u = 0; u < TS; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = acc[u][e];
          if constexpr (COPIES >= 2) x = copy == 1 ? acc[TS + u][e] : x;
          if constexpr (COPIES == 4) x = copy == 2 ? acc[2][e] : copy == 3 ? acc[3][e] : x;
          sc[u][e] = x * a.c2;
        }
      if (~ok) {                                         // some keys are not seen
#pragma unroll
        for (int u = 0; u < TS; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((ok >> (16 * (TS * copy + u) + 4 * grp + e)) & 1ull)) sc[u][e] = -INFINITY;
        // their rows of V are zero, whatever lies in the cache
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (!((ok >> (16 * t + c16)) & 1ull)) {
#pragma unroll
            for (int j = 0; j < NKS; ++j) vr.x[t][j] = 0;
            vr.scale[t] = 127;
          }
      }
      if constexpr (SCORES) {
        if (head < gn) {
          float* row = a.scores + ((size_t)now.s * a.Hq + h0 + head) * a.score_stride;
#pragma unroll
          for (int u = 0; u < TS; ++u) {
            const long long key = (long long)now.tl.tile(i) * FT + 16 * (TS * copy + u) + 4 * grp;
            if (key < a.score_stride) *reinterpret_cast<v4f*>(row + key) = v4f{sc[u][0], sc[u][1], sc[u][2], sc[u][3]};
          }
        }
      }
      float x = sc[0][0];
#pragma unroll
      for (int e = 1; e < 4 * TS; ++e) x = smax(x, sc[e >> 2][e & 3]);
      if constexpr (COPIES >= 2) x = smax(x, __int_as_float(dpp<kTurn + 8>(__float_as_int(x))));
      if constexpr (COPIES == 4) x = smax(x, __int_as_float(dpp<kTurn + 4>(__float_as_int(x))));
      const float m_new = smax(m, max_over_groups(x));
      const float mc = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - mc);
      m = m_new;
      float sum = 0.0f;
      uint32_t hi[2 * TS], lo[2 * TS];                   // P's upper part, and what its rounding left
#pragma unroll
      for (int e = 0; e < 4 * TS; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(sc[e >> 2][e & 3] - mc), p1 = __builtin_amdgcn_exp2f(sc[e >> 2][(e & 3) + 1] - mc);
        sum += p0 + p1;
        hi[e / 2] = pack16<true>(p0, p1);
        lo[e / 2] = pack16<true>(p0 - bf16_to_f32((uint16_t)hi[e / 2]), p1 - bf16_to_f32((uint16_t)(hi[e / 2] >> 16)));
      }
      l = l * alpha + sum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int e = 0; e < 4; ++e) oacc[db][e] *= alpha;
      }
      // the product's columns of the first copy: its own keys, and those of the other copies
      v4i pk[2], pl[2];                                  // keys 32 h + 16 (j / 2) + 4 grp + ...
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        auto put = [&](auto T_, uint32_t h, uint32_t g) {
          constexpr int t = decltype(T_)::value;
          pk[t / 2][2 * (t & 1) + w] = (int)h;
          pl[t / 2][2 * (t & 1) + w] = (int)g;
        };
        if constexpr (COPIES == 4) {
          put(ic<0>{}, hi[w], lo[w]);
          put(ic<1>{}, dpp<kLanesOn + 4>(hi[w]), dpp<kLanesOn + 4>(lo[w]));
          put(ic<2>{}, dpp<kLanesOn + 8>(hi[w]), dpp<kLanesOn + 8>(lo[w]));
          put(ic<3>{}, dpp<kLanesOn + 12>(hi[w]), dpp<kLanesOn + 12>(lo[w]));
        } else if constexpr (COPIES == 2) {
          put(ic<0>{}, hi[w], lo[w]);
          put(ic<1>{}, hi[2 + w], lo[2 + w]);
          put(ic<2>{}, dpp<kLanesOn + 8>(hi[w]), dpp<kLanesOn + 8>(lo[w]));
          put(ic<3>{}, dpp<kLanesOn + 8>(hi[2 + w]), dpp<kLanesOn + 8>(lo[2 + w]));
        } else {
          put(ic<0>{}, hi[w], lo[w]);
          put(ic<1>{}, hi[2 + w], lo[2 + w]);
          put(ic<2>{}, hi[4 + w], lo[4 + w]);
          put(ic<3>{}, hi[6 + w], lo[6 + w]);
        }
      }
      // V through the wave's tile, 32 keys at a time
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t va = opaque(vat);
      static_for<2>([&](auto H_) {
        constexpr int h = decltype(H_)::value;
        const uint32_t wa = opaque(wat);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float f = __uint_as_float((uint32_t)vr.scale[2 * h + t] << 23);
#pragma unroll
          for (int j = 0; j < NKS; ++j)
            *(__attribute__((address_space(3))) v4i*)(uintptr_t)((wa ^ (16 * j)) + 16 * ROW * t) = widen_fp4(vr.x[2 * h + t][j], f);
        }
        if constexpr (h == 1 && WHOLE) load(now, i + FW, o, v_buf, vs_buf, vr);
        else if constexpr (h == 1) load_each(now, i + FW, at1, v_rows, a.c.vs, v_scale, vr);
#pragma unroll
        for (int d4 = 0; d4 < NDB; d4 += 4) {
          __builtin_amdgcn_sched_barrier(0);
          v4i x[4];                                      // 32 keys of 4 channel blocks: two reads each, 16 keys apart
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t at = va ^ (32 * (d4 + d));
            const v2u lower = tr_read(at), upper = tr_read(at + 16 * ROW);
            x[d] = v4i{(int)lower[0], (int)lower[1], (int)upper[0], (int)upper[1]};
          }
#pragma unroll
          for (int d = 0; d < 4; ++d) oacc[d4 + d] = mma16<true>(x[d], pl[h], oacc[d4 + d]);
#pragma unroll
          for (int d = 0; d < 4; ++d) oacc[d4 + d] = mma16<true>(x[d], pk[h], oacc[d4 + d]);
        }
      });
      at = at1;
      at1 = at2;
    }

    // join the copies and the waves
    if constexpr (COPIES >= 2) l += __int_as_float(dpp<kTurn + 8>(__float_as_int(l)));
    if constexpr (COPIES == 4) l += __int_as_float(dpp<kTurn + 4>(__float_as_int(l)));
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    float* const ml = reinterpret_cast<float*>(lds + FW * REG);
    if (grp == 0 && copy == 0) {
      ml[(wave * DG + head) * 2] = m;
      ml[(wave * DG + head) * 2 + 1] = l;
    }
    lds_barrier();                                       // (the next part's rows stay in flight)
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < FW; ++w) mm = smax(mm, ml[(w * DG + head) * 2]);
    const float mc = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < FW; ++w) ll += ml[(w * DG + head) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * DG + head) * 2] - mc);
    const float f = __builtin_amdgcn_exp2f(m - mc);
    if (copy == 0) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        *reinterpret_cast<v4f*>(vt + (head * PADQ + 16 * db + 4 * grp) * 4) = oacc[db] * v4f{f, f, f, f};
    }
    lds_barrier();

    const bool whole = now.off == 0 && now.cnt == now.steps;
    const size_t slot = (size_t)blockIdx.x * 2 + (now.off == 0 ? 1 : 0);
    if (wave == 0 && grp == 0 && c16 < gn) {
      if (whole) {
        const float l2 = ll > 0.0f || ll != ll ? mm + __builtin_log2f(ll) : -INFINITY;
        if (a.lse) a.lse[(size_t)s * a.Hq + h0 + c16] = l2 * 0.69314718055994530942f;
        if (SCORES) a.lse2[(size_t)s * a.Hq + h0 + c16] = l2;
      } else {
        float* p = a.part + (size_t)a.nw * 2 * a.Hq * D + (slot * a.Hq + h0 + c16) * 2;
        p[0] = mm;
        p[1] = ll;
      }
    }
    // thread: head tid / 16, 4 channels at a time
    const int qh = tid >> 4;
    const float lq = __shfl(ll, qh % HC, 64);            // lane qh holds head qh's sum
    if (qh < gn) {
      const float inv = lq > 0.0f || lq != lq ? 1.0f / lq : 0.0f;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const int d = 64 * c + 4 * (tid & 15);
        v4f x = v4f{};
#pragma unroll
        for (int w = 0; w < FW; ++w) x += *reinterpret_cast<const v4f*>(lds + w * REG + (qh * PADQ + d) * 4);
        if (whole) {
          const v2u o = {pack16<BF16>(x[0] * inv, x[1] * inv), pack16<BF16>(x[2] * inv, x[3] * inv)};
          *reinterpret_cast<v2u*>((uint16_t*)a.o + ((size_t)s * a.Hq + h0 + qh) * D + d) = o;
        } else {
          *reinterpret_cast<v4f*>(a.part + (slot * a.Hq + h0 + qh) * D + d) = x;
        }
      }
    }
    if (a.nw == 0) return;
    r0 += now.cnt;
    if (r0 >= r1) return;
    s = find_step(a, mine, upto, r0, &before);           // the next one that has steps
    lds_barrier();                                       // its V tiles overwrite the join's LDS
  }
}

// Sequences whose tiles several workgroups shared: O = sum O_w 2^(m_w - m) / l.  One workgroup per
// (sequence, query head); each of its waves adds up every fourth part by itself, with the maximum of
// these alone, so that nothing but the lengths is waited for before a wave's parts are on their way; the
// waves' sums are joined through LDS.  (32 sequences of up to 8000 tokens, 64 / 4 heads: the call takes
// 30.7 us, 31.8 with a common maximum first; 16 waves are no better for 64 parts, and worse for few.)
constexpr int JW = 4;                   // its waves
template <int D, bool BF16>
__global__ __launch_bounds__(64 * JW) void join_fp4_kernel(const Decode a) {
  constexpr int CL = D / 64, U = 4;                      // channels per lane; parts on their way per wave
  __shared__ float sums[JW][D + 2];
  const int s = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int mine = a.before ? 0 : steps_of_lane<FT, FW>(a), upto = a.before ? 0 : lanes_up_to(mine);
  const Line line = steps_line(a, upto);
  const long long before = a.before ? a.before[s] : __shfl(upto - mine, s, 64);
  const int steps = a.before ? (int)(a.before[s + 1] - before) : __shfl(mine, s, 64);
  const int w0 = steps > 0 ? (int)divide(before, line.share) : 0, w1 = steps > 0 ? (int)divide(before + steps - 1, line.share) : -1;
  if (w0 == w1) return;                                  // final already
  const float* ml = a.part + (size_t)a.nw * 2 * a.Hq * D;
  float m = -INFINITY, l = 0.0f, x[CL] = {};
  for (int w = w0 + wave; w <= w1; w += U * JW) {
    float mw[U], lw[U], p[U][CL], top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = imin(w + u * JW, w1);
      // a share's slot 1 if the sequence begins in it, slot 0 if it began before
      const size_t k = ((size_t)at * 2 + (at == w0 ? 1 : 0)) * a.Hq + h;
      mw[u] = ml[k * 2];
      lw[u] = ml[k * 2 + 1];
#pragma unroll
      for (int i = 0; i < CL; ++i) p[u][i] = a.part[k * D + lane * CL + i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) top = smax(top, mw[u]);
    const float mc = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - mc);
    m = top;
    l *= f;
#pragma unroll
    for (int i = 0; i < CL; ++i) x[i] *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float g = w + u * JW <= w1 ? __builtin_amdgcn_exp2f(mw[u] - mc) : 0.0f;
      l += lw[u] * g;
#pragma unroll
      for (int i = 0; i < CL; ++i) x[i] += p[u][i] * g;
    }
  }
#pragma unroll
  for (int i = 0; i < CL; ++i) sums[wave][lane * CL + i] = x[i];
  if (lane == 0) {
    sums[wave][D] = l;
    sums[wave][D + 1] = m;
  }
  __syncthreads();
  if (wave > 0) return;
  float all = -INFINITY, sum = 0.0f, o[CL] = {};
#pragma unroll
  for (int w = 0; w < JW; ++w) all = smax(all, sums[w][D + 1]);
  const float mc = all == -INFINITY ? 0.0f : all;
#pragma unroll
  for (int w = 0; w < JW; ++w) {
    const float f = __builtin_amdgcn_exp2f(sums[w][D + 1] - mc);
    sum += sums[w][D] * f;
#pragma unroll
    for (int i = 0; i < CL; ++i) o[i] += sums[w][lane * CL + i] * f;
  }
  const bool some = sum > 0.0f || sum != sum;
  const float inv = some ? 1.0f / sum : 0.0f;
  uint16_t* out = (uint16_t*)a.o + ((size_t)s * a.Hq + h) * D + lane * CL;
  if constexpr (D == 128) *reinterpret_cast<uint32_t*>(out) = pack16<BF16>(o[0] * inv, o[1] * inv);
  else *out = (uint16_t)pack16<BF16>(o[0] * inv, 0.0f);
  if (lane == 0) {
    const float l2 = some ? all + __builtin_log2f(sum) : -INFINITY;
    if (a.lse) a.lse[(size_t)s * a.Hq + h] = l2 * 0.69314718055994530942f;
    if (a.lse2) a.lse2[(size_t)s * a.Hq + h] = l2;
  }
}

template <int D, bool BF16>
hipError_t launch_t(const Decode& a, hipStream_t st) {
  const int G = a.Hq / a.c.Hkv;
  const dim3 grid((unsigned)(a.nw > 0 ? a.nw : a.c.S), (unsigned)a.c.Hkv, (unsigned)cdiv(G, DG)), block(64 * FW);
  hipError_t e = hipSuccess;
  if (a.before) {
    hipLaunchKernelGGL((line_kernel<FT, FW>), dim3(1), dim3(1024), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  // (the buffers' bounds, 2^31 bytes, hold for a load's whole offset; a lane's own of 2^31 marks one that is none)
  const Strides &ks = a.c.ks, &vs = a.c.vs;
  const double most = (a.c.pages - 1.0) * ks.b + (a.c.page_size - 1.0) * ks.n + D / 2, rows = (double)a.c.pages * a.c.Hkv * a.c.page_size;
  const bool whole = a.c.page_size % 16 == 0 && ks.b == vs.b && ks.n == vs.n && ks.n < 1LL << 27 && most <= 0x1p31 &&
                     rows * (D / 32) <= 0x1p31;
#define SAGE_DECODE_FP4(WHOLE, SCORES)                                                                                      \
  if (G <= 4) hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 4, WHOLE, SCORES>), grid, block, 0, st, a);              \
  else if (G <= 8) hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 2, WHOLE, SCORES>), grid, block, 0, st, a);         \
  else hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 1, WHOLE, SCORES>), grid, block, 0, st, a)
  if (whole && a.weights) { SAGE_DECODE_FP4(true, true); }
  else if (whole) { SAGE_DECODE_FP4(true, false); }
  else if (a.weights) { SAGE_DECODE_FP4(false, true); }
  else { SAGE_DECODE_FP4(false, false); }
#undef SAGE_DECODE_FP4
  e = hipGetLastError();
  if (e == hipSuccess && a.nw > 0) {
    hipLaunchKernelGGL((join_fp4_kernel<D, BF16>), dim3((unsigned)a.c.S, (unsigned)a.Hq), dim3(64 * JW), 0, st, a);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.weights) e = launch_add_weights(a, st);
  return e;
}

}  // namespace

// As decode_workgroups (never more than it: the same workspace does), for longer steps.  (Shares cut at
// single tiles are more even, but begin and end more parts: 32 x 8000 tokens, D = 64: 41 -> 44 us.)
int decode_fp4_workgroups(int S, int Hq, int Hkv, int capacity) {
  const long long steps = cdiv(capacity, FT * FW) + 1;
  if (steps <= 5) return 0;
  const int heads = Hkv * cdiv(Hq / Hkv, DG);
  const long long want = imax(1, 512 / heads), most = (long long)S * steps;
  return (int)(want < most ? want : most);
}

hipError_t launch_paged_decode_fp4(const Decode& a, int D, bool bf16, hipStream_t st) {
  if (D == 128) return bf16 ? launch_t<128, true>(a, st) : launch_t<128, false>(a, st);
  return bf16 ? launch_t<64, true>(a, st) : launch_t<64, false>(a, st);
}

}  // namespace sage
