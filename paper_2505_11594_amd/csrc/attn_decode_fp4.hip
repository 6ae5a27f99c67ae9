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
// A group of up to 4 (8) query heads leaves 12 (8) of the product's 16 columns free: its
// heads stand there 4 (2) times, and each copy takes the softmax of another 16 (32) of
// the tile's 64 keys.  P is brought together again within the rows of 16 lanes.
#include "decode_split.h"

namespace sage {

namespace {

constexpr int FT = 64;                  // keys per tile

// 8 values of q in bf16: rounded, and of fp16 what the rounding left (11 bits in 8 and 8: exact).
template <bool BF16>
__device__ __forceinline__ void split_q(const uint16_t* q, v4i* hi, v4i* lo) {
  const v4i v = *reinterpret_cast<const v4i*>(q);
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

template <int D, bool BF16, int COPIES>
__global__ __launch_bounds__(64 * DW, 2) void paged_decode_fp4_kernel(const Decode a) {
  constexpr int ROW = D * 2, SB = D / 32;                // bytes of a V row in LDS; scale bytes of a cached row
  constexpr int HC = 16 / COPIES, TS = 4 / COPIES;       // heads per copy; subtiles of 16 keys whose softmax a copy takes
  constexpr int NKS = D / 32;                            // steps of 32 channels of S; lane: 8 channels of each, D / 4 in a row
  constexpr int VL = D / 32, NDB = D / 16;
  constexpr int PADQ = D + 4;
  constexpr int REG = FT * ROW;                          // LDS bytes per wave: V tile, then its O
  static_assert(REG >= DG * PADQ * 4 && REG % 256 == 0, "O fits; addresses inside a tile are xor-ed");
  __shared__ __attribute__((aligned(256))) uint8_t lds[DW * REG + DW * DG * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, grp = lane >> 4, copy = c16 / HC, head = c16 % HC;
  const int hk = blockIdx.y, G = a.Hq / a.c.Hkv, g0 = blockIdx.z * DG, gn = imin(DG, G - g0);
  const int h0 = hk * G + g0;                            // first query head
  uint8_t* const vt = lds + wave * REG;
  const uint32_t vbase = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)vt;
  const uint32_t vat = vbase + (4 * grp + c16 / 4) * ROW + vswz<D>(4 * grp + c16 / 4, (c16 & 3) / 2) * 16 + 8 * (c16 & 1);
  const uint8_t* const k_scale = (const uint8_t*)a.c.k_scale;
  const uint8_t* const v_scale = (const uint8_t*)a.c.v_scale;

  long long r0 = 0, r1 = 0, before = 0;
  int s = blockIdx.x, mine = 0, upto = 0;
  if (a.nw > 0) {
    if (!a.before) {
      mine = steps_of_lane<FT>(a);
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
    const TileList tl = seq_tiles<FT>(a, s, &n);
    const int steps = cdiv(tl.count, DW);
    const int off = a.nw > 0 ? (int)(r0 - before) : 0;
    const int cnt = a.nw > 0 ? (int)min((long long)(steps - off), r1 - r0) : steps;
    const int tend = imin(tl.count, DW * (off + cnt));
    const int32_t* const table = a.c.table + (size_t)s * a.c.max_pages;

    v4i qreg[NKS], qrest[BF16 ? 1 : NKS];                // channels in the order in which K's lie in its registers
    {
      const uint16_t* q = (const uint16_t*)a.q + s * a.q_s + (h0 + imin(head, gn - 1)) * a.q_h + D / 4 * grp;
#pragma unroll
      for (int j = 0; j < NKS; ++j) split_q<BF16>(q + 8 * j, &qreg[j], &qrest[BF16 ? 0 : j]);
    }
    v4f oacc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = v4f{};
    float m = -INFINITY, l = 0.0f;                       // m in log2 units

    // the page of this lane's key (key `lane` of a tile), -1 where it has none
    auto page_of = [&](int i) -> int {
      const int key = tl.tile(i) * FT + lane;
      if (i >= tend || !decode_sees(key, n, a.window, a.sinks)) return -1;
      const int id = table[key / ps];
      return page_ok(id, a.c.pages) ? id : -1;
    };
    struct Rows {
      int k[4][NKS];                                     // K: key 16 t + c16, channels from D / 4 grp on
      v4i v[VL];                                         // V: key 64 / VL j + lane / SB, channels from 32 (lane % SB) on
      int ks[4], vs[VL];
    };
    auto load = [&](int i, int id, Rows& r) {
      const int key = tl.tile(i) * FT + lane;
      const int pid = imax(id, 0), slot = id >= 0 ? key % ps : 0;        // keys without a page: the cache's first row
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int p = __shfl(pid, 16 * t + c16, 64), sl = __shfl(slot, 16 * t + c16, 64);
        const uint8_t* k = (const uint8_t*)a.c.k + (p * a.c.ks.b + hk * a.c.ks.h + sl * a.c.ks.n) + D / 8 * grp;
        if constexpr (D == 128) *reinterpret_cast<v4i*>(r.k[t]) = *reinterpret_cast<const v4i*>(k);
        else *reinterpret_cast<v2u*>(r.k[t]) = *reinterpret_cast<const v2u*>(k);
        r.ks[t] = k_scale[(((size_t)p * a.c.Hkv + hk) * ps + sl) * SB + D * grp / 128];
      }
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int row = 64 / SB * j + lane / SB, ch = lane % SB;
        const int p = __shfl(pid, row, 64), sl = __shfl(slot, row, 64);
        r.v[j] = *reinterpret_cast<const v4i*>((const uint8_t*)a.c.v + (p * a.c.vs.b + hk * a.c.vs.h + sl * a.c.vs.n) + 16 * ch);
        r.vs[j] = v_scale[(((size_t)p * a.c.Hkv + hk) * ps + sl) * SB + ch];
      }
    };

    int i = DW * off + wave;
    int id = page_of(i), id1 = page_of(i + DW);
    Rows cur, nxt;
    if (i < tend) load(i, id, cur);
    for (; i < tend; i += DW) {
      const int id2 = page_of(i + 2 * DW);
      if (i + DW < tend) load(i + DW, id1, nxt);
      const unsigned long long ok = __builtin_amdgcn_ballot_w64(id >= 0);    // bit: key of the tile

      // scores of keys 16 t + 4 grp + e, of which this lane takes t = TS copy + u
      v4f acc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float f = __uint_as_float((uint32_t)cur.ks[t] << 23);
        acc[t] = v4f{};
#pragma unroll
        for (int j = 0; j < NKS; ++j) {
          const v4i k = widen_fp4(cur.k[t][j], f);
          if constexpr (!BF16) acc[t] = mma16<true>(k, qrest[j], acc[t]);
          acc[t] = mma16<true>(k, qreg[j], acc[t]);
        }
      }
      float sc[TS][4];
#pragma unroll
      for (int u = 0; u < TS; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = acc[u][e];
          if constexpr (COPIES >= 2) x = copy == 1 ? acc[TS + u][e] : x;
          if constexpr (COPIES == 4) x = copy == 2 ? acc[2][e] : copy == 3 ? acc[3][e] : x;
          const int key = 16 * (TS * copy + u) + 4 * grp + e;
          sc[u][e] = (ok >> key) & 1ull ? x * a.c2 : -INFINITY;
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
      // V into the wave's tile; rows that are not seen are zero, whatever lies in the cache
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int row = 64 / SB * j + lane / SB, ch = lane % SB;
        v4i v = cur.v[j];
        uint32_t f = (uint32_t)cur.vs[j] << 23;
        if (!((ok >> row) & 1ull)) { v = v4i{}; f = 0x3F800000u; }
#pragma unroll
        for (int w = 0; w < 4; ++w)
          *reinterpret_cast<v4i*>(vt + row * ROW + vswz<D>(row, 4 * ch + w) * 16) = widen_fp4(v[w], __uint_as_float(f));
      }
      const uint32_t va = opaque(vat);
      static_for<2 * NDB / 4>([&](auto B_) {
        constexpr int b4 = 4 * (decltype(B_)::value % (NDB / 4)), h = decltype(B_)::value / (NDB / 4);
        v8bf vv[4];                                      // 32 keys of 4 channel blocks: two reads each, 16 keys apart
        vt_read4<32 * h * ROW, (32 * h + 16) * ROW>(va ^ (32 * b4), va ^ (32 * b4 + 32), va ^ (32 * b4 + 64), va ^ (32 * b4 + 96),
                                                    vv[0], vv[1], vv[2], vv[3]);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const v4i x = __builtin_bit_cast(v4i, vv[d]);
          oacc[b4 + d] = mma16<true>(x, pl[h], mma16<true>(x, pk[h], oacc[b4 + d]));
        }
      });
      id = id1;
      id1 = id2;
      cur = nxt;
    }

    // join the copies and the 4 waves
    if constexpr (COPIES >= 2) l += __int_as_float(dpp<kTurn + 8>(__float_as_int(l)));
    if constexpr (COPIES == 4) l += __int_as_float(dpp<kTurn + 4>(__float_as_int(l)));
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    float* const ml = reinterpret_cast<float*>(lds + DW * REG);
    if (grp == 0 && copy == 0) {
      ml[(wave * DG + head) * 2] = m;
      ml[(wave * DG + head) * 2 + 1] = l;
    }
    __syncthreads();                                     // also: every wave is past its last V tile
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < DW; ++w) mm = smax(mm, ml[(w * DG + head) * 2]);
    const float mc = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < DW; ++w) ll += ml[(w * DG + head) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * DG + head) * 2] - mc);
    const float f = __builtin_amdgcn_exp2f(m - mc);
    if (copy == 0) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        *reinterpret_cast<v4f*>(vt + (head * PADQ + 16 * db + 4 * grp) * 4) = oacc[db] * v4f{f, f, f, f};
    }
    __syncthreads();

    const bool whole = off == 0 && cnt == steps;
    const size_t slot = (size_t)blockIdx.x * 2 + (off == 0 ? 1 : 0);
    if (wave == 0 && grp == 0 && c16 < gn) {
      if (whole) {
        const float l2 = ll > 0.0f || ll != ll ? mm + __builtin_log2f(ll) : -INFINITY;
        if (a.lse) a.lse[(size_t)s * a.Hq + h0 + c16] = l2 * 0.69314718055994530942f;
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
        for (int w = 0; w < DW; ++w) x += *reinterpret_cast<const v4f*>(lds + w * REG + (qh * PADQ + d) * 4);
        if (whole) {
          const v2u o = {pack16<BF16>(x[0] * inv, x[1] * inv), pack16<BF16>(x[2] * inv, x[3] * inv)};
          *reinterpret_cast<v2u*>((uint16_t*)a.o + ((size_t)s * a.Hq + h0 + qh) * D + d) = o;
        } else {
          *reinterpret_cast<v4f*>(a.part + (slot * a.Hq + h0 + qh) * D + d) = x;
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

template <int D, bool BF16>
hipError_t launch_t(const Decode& a, hipStream_t st) {
  const int G = a.Hq / a.c.Hkv;
  const dim3 grid((unsigned)(a.nw > 0 ? a.nw : a.c.S), (unsigned)a.c.Hkv, (unsigned)cdiv(G, DG)), block(64 * DW);
  hipError_t e = hipSuccess;
  if (a.before) {
    hipLaunchKernelGGL(line_kernel<FT>, dim3(1), dim3(1024), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (G <= 4) hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 4>), grid, block, 0, st, a);
  else if (G <= 8) hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 2>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_decode_fp4_kernel<D, BF16, 1>), grid, block, 0, st, a);
  e = hipGetLastError();
  if (e == hipSuccess && a.nw > 0) {
    hipLaunchKernelGGL((join_kernel<D, BF16, FT>), dim3((unsigned)a.c.S, (unsigned)a.Hq), dim3(256), 0, st, a, 0.0f);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// As decode_workgroups (never more than it: the same workspace does), for steps of 64-key tiles.
int decode_fp4_workgroups(int S, int Hq, int Hkv, int capacity) {
  const long long steps = cdiv(capacity, FT * DW) + 1;
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
