// C ABI of the window attention, the norms of queries and keys with their rotation, the
// paged cache, one-token attention over it, and page tables.
// Argument checks run on the host before any HIP call; kernels are enqueued on the
// caller's stream; nothing is allocated.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "lm_args.h"
#include "rows.h"
#include "sage_mi355x.h"

namespace {

using sage::Strides;

constexpr long long kMaxElems = 1LL << 40;     // bound on B*H*N*D, and on every stride
constexpr long long kMaxRowStride = 1LL << 22; // token stride of a tensor that is read in tiles (32-bit offsets inside one)
constexpr int kMaxHeads = 65535, kMaxSeqs = 65535;   // launch grid limits
constexpr int kMaxCapacity = 1 << 30;

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline float softmax_c2(int D) { return (float)(1.0 / (std::log(2.0) * std::sqrt((double)D))); }
inline int hip_status(hipError_t e) { return e == hipSuccess ? SAGE_OK : SAGE_ERR_HIP; }
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

inline Strides strides_or(const sage_strides* s, int H, int N, int D) {
  if (s) return Strides{s->b, s->h, s->n};
  return Strides{(long long)H * N * D, (long long)N * D, D};
}
// Rows of D channels start on 16 bytes (`per` elements of them).
inline bool strides_ok(const Strides& s, int per, long long max_n) {
  for (long long x : {s.b, s.h, s.n})
    if (x < 0 || x > kMaxElems || x % per) return false;
  return s.n <= max_n;
}
// No two rows of a written tensor overlap (a sufficient condition: sorted by
// stride, each dimension steps over all of the smaller ones).
inline bool distinct_rows(const Strides& s, long long nb, long long nh, long long nn, int D) {
  struct Dim { long long stride, size; } d[3] = {{s.b, nb}, {s.h, nh}, {s.n, nn}};
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  long long extent = D;
  for (const Dim& x : d) {
    if (x.size <= 1) continue;
    if (x.stride < extent || x.stride > (1LL << 62) / x.size) return false;
    extent += x.stride * (x.size - 1);
  }
  return true;
}

int check_heads(int Hq, int Hkv, int D) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv || Hq > kMaxHeads) return SAGE_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return SAGE_ERR_INVALID_ARG;
  return SAGE_OK;
}

int check_window(int B, int Hq, int Hkv, int N, int D, int window, int sinks) {
  const int rc = check_heads(Hq, Hkv, D);
  if (rc != SAGE_OK) return rc;
  if (B <= 0 || N <= 0 || window < 1 || sinks < 0) return SAGE_ERR_INVALID_ARG;
  const long long Np = ((long long)N + 127) / 128 * 128;
  if (Np * D > (1LL << 31) || (long long)B * Hq > (1LL << 30) || (long long)B * Hq * Np * D > kMaxElems)
    return SAGE_ERR_INVALID_ARG;
  if ((long long)B * Hq * (Np / 128) >= (1LL << 24)) return SAGE_ERR_INVALID_ARG;   // a workgroup of 256 each: 2^32 threads a launch
  return SAGE_OK;
}
// Where even the last query's window begins among the sinks (or is everything), every
// key is seen as without a window.
inline void clamp_window(int n, int* window, int* sinks) {
  if ((long long)*window + *sinks < n) return;
  *window = n;
  *sinks = 0;
}

// `written`: rows are stored, so they may not overlap.
int check_pages(const sage_kv_cache* c, bool written, bool fp4) {
  if (!c || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return SAGE_ERR_INVALID_ARG;
  if (!c->k_scale != !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return SAGE_ERR_INVALID_ARG;
  if (fp4 && !c->k_scale) return SAGE_ERR_INVALID_ARG;
  if (c->pages <= 0 || c->page_size <= 0 || c->page_size > kMaxCapacity) return SAGE_ERR_INVALID_ARG;
  if (check_heads(c->Hkv, c->Hkv, c->D) != SAGE_OK) return SAGE_ERR_INVALID_ARG;
  const int per = c->k_scale ? 16 : 8;
  for (const sage_strides* s : {&c->k_strides, &c->v_strides}) {
    const Strides x{s->b, s->h, s->n};
    if (!strides_ok(x, per, kMaxElems)) return SAGE_ERR_INVALID_ARG;
    if (written && !distinct_rows(x, c->pages, c->Hkv, c->page_size, fp4 ? c->D / 2 : c->D)) return SAGE_ERR_INVALID_ARG;
  }
  return SAGE_OK;
}
int check_cache(const sage_kv_cache* c, const int32_t* table, int max_pages, int S, bool written, bool fp4 = false) {
  const int rc = check_pages(c, written, fp4);
  if (rc != SAGE_OK) return rc;
  if (!table || !aligned(table, 4) || max_pages <= 0 || S <= 0 || S > kMaxSeqs) return SAGE_ERR_INVALID_ARG;
  if ((long long)max_pages * c->page_size > kMaxCapacity) return SAGE_ERR_INVALID_ARG;
  return SAGE_OK;
}
sage::Cache cache_of(const sage_kv_cache* c, const int32_t* table, int max_pages, int S) {
  sage::Cache r;
  r.k = c->k; r.v = c->v; r.k_scale = c->k_scale; r.v_scale = c->v_scale;
  r.ks = Strides{c->k_strides.b, c->k_strides.h, c->k_strides.n};
  r.vs = Strides{c->v_strides.b, c->v_strides.h, c->v_strides.n};
  r.pages = c->pages; r.page_size = c->page_size; r.Hkv = c->Hkv;
  r.table = table; r.S = S; r.max_pages = max_pages;
  return r;
}

// The arguments that norm and rotation share with their backward.
int check_norm_rope(sage::NormRope& a, const void* q, const void* k, const float* q_weight, const float* k_weight,
                    const float* inv_freq, int rotary, const int32_t* pos, int pos_per_token, const int32_t* lens, int B, int Hq,
                    int Hkv, int N, int D, float eps, unsigned flags, const sage_strides* q_strides,
                    const sage_strides* k_strides) {
  if (flags & ~(unsigned)(SAGE_IN_BF16 | SAGE_ROPE_PAIRS)) return SAGE_ERR_INVALID_ARG;
  if (check_heads(Hq, Hkv, D) != SAGE_OK || B <= 0 || N <= 0) return SAGE_ERR_INVALID_ARG;
  if ((long long)B * N > (1LL << 30) || (long long)B * N * Hq * D > kMaxElems) return SAGE_ERR_INVALID_ARG;
  if (rotary < 0 || rotary > D || rotary % 8 || (rotary > 0 && !inv_freq) || pos_per_token < 0 || pos_per_token > 1)
    return SAGE_ERR_INVALID_ARG;
  if (!(eps >= 0x1p-100f) || !(eps <= 1.0f)) return SAGE_ERR_INVALID_ARG;
  if (!q || !k || !aligned(q, 16) || !aligned(k, 16)) return SAGE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)q_weight, (const void*)k_weight, (const void*)inv_freq, (const void*)pos, (const void*)lens})
    if (!aligned(p, 4)) return SAGE_ERR_INVALID_ARG;
  a.q = q; a.k = k; a.wq = q_weight; a.wk = k_weight; a.freq = inv_freq; a.pos = pos; a.lens = lens;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.N = N; a.R = rotary; a.pos_each = pos_per_token; a.eps = eps;
  a.qs = strides_or(q_strides, Hq, N, D); a.ks = strides_or(k_strides, Hkv, N, D);
  for (const Strides& s : {a.qs, a.ks})
    if (!strides_ok(s, 8, kMaxElems)) return SAGE_ERR_INVALID_ARG;
  return SAGE_OK;
}
// Its outputs: rows apart.
int check_norm_rope_out(sage::NormRope& a, void* zq, void* zk, int D, const sage_strides* zq_strides, const sage_strides* zk_strides) {
  if (!zq || !zk || !aligned(zq, 16) || !aligned(zk, 16)) return SAGE_ERR_INVALID_ARG;
  a.zq = zq; a.zk = zk;
  a.zqs = strides_or(zq_strides, a.Hq, a.N, D); a.zks = strides_or(zk_strides, a.Hkv, a.N, D);
  for (const Strides& s : {a.zqs, a.zks})
    if (!strides_ok(s, 8, kMaxElems)) return SAGE_ERR_INVALID_ARG;
  if (!distinct_rows(a.zqs, a.B, a.Hq, a.N, D) || !distinct_rows(a.zks, a.B, a.Hkv, a.N, D)) return SAGE_ERR_INVALID_ARG;
  return SAGE_OK;
}
// No output has memory in common with another tensor, but for that of its own heads (zq with q and gq, zk with k and
// gk) where it is the very same: a wave stores a row when it has read it, and nobody else reads it.  Any other row
// of an input may still be waiting for its wave.
bool norm_rope_apart(const sage::NormRope& a, int D) {
  struct View { const void* p; const Strides* s; int H; };
  const View zq{a.zq, &a.zqs, a.Hq}, zk{a.zk, &a.zks, a.Hkv}, q[2] = {{a.q, &a.qs, a.Hq}, {a.gq, &a.gqs, a.Hq}},
             k[2] = {{a.k, &a.ks, a.Hkv}, {a.gk, &a.gks, a.Hkv}};
  auto meet = [&](const View& x, const View& y) {
    const sage::RowSet rx(D, x.s->b, a.B, x.s->h, x.H, x.s->n, a.N), ry(D, y.s->b, a.B, y.s->h, y.H, y.s->n, a.N);
    int steps = 4096;
    return sage::rows_meet(rx, 0, ry, 0, ((long long)(intptr_t)y.p - (long long)(intptr_t)x.p) / 2, &steps);
  };
  auto same = [&](const View& x, const View& y) {
    return x.p == y.p && (a.B == 1 || x.s->b == y.s->b) && (x.H == 1 || x.s->h == y.s->h) && (a.N == 1 || x.s->n == y.s->n);
  };
  if (meet(zq, zk)) return false;
  for (int i = 0; i < 2 && q[i].p; ++i)
    if ((!same(zq, q[i]) && meet(zq, q[i])) || (!same(zk, k[i]) && meet(zk, k[i])) || meet(zq, k[i]) || meet(zk, q[i])) return false;
  return true;
}

struct BwdWs {
  size_t lb, delta, norms, scales, part, mpart, total;
  int chunks, mchunks, mshare;
};
BwdWs bwd_ws(int B, int Hq, int Hkv, int N, int D, int window, int sinks) {
  BwdWs w;
  w.chunks = sage::window_bwd_chunks(B, Hq, Hkv, N, sinks);
  w.mshare = sage::window_bwd_share(B, Hq, Hkv, N, window, &w.mchunks);
  size_t off = 0;
  const size_t rows = up256(sage::window_bwd_row_floats(B, Hq, N) * sizeof(float));
  w.lb = off; off += rows;
  w.delta = off; off += rows;
  w.norms = off; off += up256(sage::window_bwd_norm_floats(B, Hq, Hkv, N) * sizeof(float));
  w.scales = off; off += up256((size_t)B * Hkv * sizeof(float));
  w.part = off; off += up256(sage::window_bwd_part_floats(B, Hq, Hkv, N, D, sinks) * sizeof(float));
  w.mpart = off; off += up256(sage::window_bwd_mpart_floats(B, Hkv, N, D, w.mchunks) * sizeof(float));
  w.total = off;
  return w;
}

struct DecodeWs {
  size_t part, line, lse2, scores, total;
  long long score_stride;
};
DecodeWs decode_ws(int S, int Hq, int Hkv, int D, int capacity, bool weights) {
  DecodeWs w;
  size_t off = 0;
  w.score_stride = (capacity + 31LL) / 32 * 32;
  w.part = off; off += up256(sage::decode_part_floats(S, Hq, Hkv, D, capacity) * sizeof(float));
  w.line = off; off += up256(sage::decode_line_longs(S, Hq, Hkv, capacity) * sizeof(long long));
  w.lse2 = off; off += weights ? up256((size_t)S * Hq * sizeof(float)) : 0;
  w.scores = off; off += weights ? up256((size_t)S * Hq * w.score_stride * sizeof(float)) : 0;
  w.total = off;
  return w;
}

int evict(const sage_kv_cache* cache, const int32_t* table, int max_pages, const int32_t* lens, const float* weights,
          int64_t weights_stride, const int32_t* new_table, int new_max_pages, int budget, int keep_first, int keep_last,
          int32_t* new_lens, float* new_weights, int32_t* kept, int S, void* workspace, size_t workspace_bytes, bool fp4,
          hipStream_t stream) {
  const int rc = check_cache(cache, table, max_pages, S, true, fp4);
  if (rc != SAGE_OK) return rc;
  if (!lens || !weights || !new_table || !new_lens || !new_weights || !kept) return SAGE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)lens, (const void*)weights, (const void*)new_table, (const void*)new_lens,
                        (const void*)new_weights, (const void*)kept})
    if (!aligned(p, 4)) return SAGE_ERR_INVALID_ARG;
  if (budget < 1 || keep_first < 0 || keep_last < 0 || (long long)keep_first + keep_last > budget) return SAGE_ERR_INVALID_ARG;
  if (new_max_pages <= 0 || (long long)new_max_pages * cache->page_size > kMaxCapacity ||
      (long long)new_max_pages * cache->page_size < budget || weights_stride < (long long)max_pages * cache->page_size)
    return SAGE_ERR_INVALID_ARG;
  // outputs that other workgroups still read would change under them
  if (new_lens == lens || new_weights == weights) return SAGE_ERR_INVALID_ARG;
  const size_t need = sage_kv_evict_workspace_size(S, cache->Hkv, max_pages, cache->page_size);
  if (need > 0) {
    if (!workspace || !aligned(workspace, 256)) return SAGE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SAGE_ERR_WORKSPACE;
  }
  sage::Evict a;
  a.hist = static_cast<int*>(workspace);
  a.c = cache_of(cache, table, max_pages, S);
  a.lens = lens; a.new_table = new_table; a.weights = weights; a.new_weights = new_weights;
  a.new_lens = new_lens; a.kept = kept; a.wstride = weights_stride;
  a.new_wstride = (long long)new_max_pages * cache->page_size;
  a.new_max_pages = new_max_pages; a.budget = budget; a.keep_first = keep_first; a.keep_last = keep_last;
  return hip_status(sage::launch_kv_evict(a, cache->D, fp4, stream));
}

}  // namespace

extern "C" {

int sage_attn_window_fwd(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* lens,
                         int B, int Hq, int Hkv, int N, int D, int window, int sinks, unsigned flags,
                         const sage_strides* q_strides, const sage_strides* k_strides, const sage_strides* v_strides,
                         const sage_strides* o_strides, hipStream_t stream) {
  if (flags & ~(unsigned)SAGE_IN_BF16) return SAGE_ERR_INVALID_ARG;
  const int rc = check_window(B, Hq, Hkv, N, D, window, sinks);
  if (rc != SAGE_OK) return rc;
  if (!q || !k || !v || !o) return SAGE_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)o})
    if (!aligned(p, 16)) return SAGE_ERR_INVALID_ARG;
  if (!aligned(lse, 4) || !aligned(lens, 4)) return SAGE_ERR_INVALID_ARG;
  sage::WindowFwd a;
  a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse; a.lens = lens;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.N = N; a.window = window; a.sinks = sinks;
  a.qs = strides_or(q_strides, Hq, N, D); a.ks = strides_or(k_strides, Hkv, N, D);
  a.vs = strides_or(v_strides, Hkv, N, D); a.os = strides_or(o_strides, Hq, N, D);
  for (const Strides& s : {a.qs, a.ks, a.vs, a.os})
    if (!strides_ok(s, 8, kMaxRowStride)) return SAGE_ERR_INVALID_ARG;
  if (!distinct_rows(a.os, B, Hq, N, D)) return SAGE_ERR_INVALID_ARG;
  a.c2 = softmax_c2(D);
  clamp_window(N, &a.window, &a.sinks);
  return hip_status(sage::launch_window_fwd(a, D, (flags & SAGE_IN_BF16) != 0, stream));
}

size_t sage_attn_window_bwd_workspace_size(int B, int Hq, int Hkv, int N, int D, int window, int sinks) {
  if (check_window(B, Hq, Hkv, N, D, window, sinks) != SAGE_OK) return 0;
  clamp_window(N, &window, &sinks);
  return bwd_ws(B, Hq, Hkv, N, D, window, sinks).total;
}

int sage_attn_window_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* dout,
                         const int32_t* lens, void* dq, void* dk, void* dv, int B, int Hq, int Hkv, int N, int D,
                         int window, int sinks, unsigned flags, const sage_strides* q_strides,
                         const sage_strides* k_strides, const sage_strides* v_strides, const sage_strides* o_strides,
                         const sage_strides* dout_strides, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (flags & ~(unsigned)SAGE_IN_BF16) return SAGE_ERR_INVALID_ARG;
  const int rc = check_window(B, Hq, Hkv, N, D, window, sinks);
  if (rc != SAGE_OK) return rc;
  if (!lse || !aligned(lse, 4) || !aligned(lens, 4)) return SAGE_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, o, dout, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!p || !aligned(p, 16)) return SAGE_ERR_INVALID_ARG;
  if ((long long)B * (Hq + Hkv) > 65535) return SAGE_ERR_INVALID_ARG;
  sage::WindowBwd a;
  a.q = q; a.k = k; a.v = v; a.o = o; a.dout = dout; a.lse = lse; a.lens = lens; a.dq = dq; a.dk = dk; a.dv = dv;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.N = N; a.window = window; a.sinks = sinks;
  a.qs = strides_or(q_strides, Hq, N, D); a.ks = strides_or(k_strides, Hkv, N, D);
  a.vs = strides_or(v_strides, Hkv, N, D); a.os = strides_or(o_strides, Hq, N, D);
  a.gs = strides_or(dout_strides, Hq, N, D);
  for (const Strides& s : {a.qs, a.ks, a.vs, a.os, a.gs})
    if (!strides_ok(s, 8, kMaxRowStride)) return SAGE_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256)) return SAGE_ERR_INVALID_ARG;
  clamp_window(N, &a.window, &a.sinks);
  const BwdWs w = bwd_ws(B, Hq, Hkv, N, D, a.window, a.sinks);
  if (workspace_bytes < w.total) return SAGE_ERR_WORKSPACE;
  uint8_t* base = static_cast<uint8_t*>(workspace);
  a.lb = reinterpret_cast<float*>(base + w.lb);
  a.delta = reinterpret_cast<float*>(base + w.delta);
  a.norms = reinterpret_cast<float*>(base + w.norms);
  a.scales = reinterpret_cast<float*>(base + w.scales);
  a.part = reinterpret_cast<float*>(base + w.part);
  a.mpart = reinterpret_cast<float*>(base + w.mpart);
  a.chunks = w.chunks; a.mchunks = w.mchunks; a.mshare = w.mshare;
  a.c2 = softmax_c2(D);
  a.rsd = (float)(1.0 / std::sqrt((double)D));
  return hip_status(sage::launch_window_bwd(a, D, (flags & SAGE_IN_BF16) != 0, stream));
}

int sage_kv_append(const sage_kv_cache* cache, const void* k, const void* v, const sage_strides* k_strides,
                   const sage_strides* v_strides, const int32_t* table, int max_pages, const int32_t* pos,
                   const int32_t* counts, float* weights, int64_t weights_stride, int S, int N, unsigned flags,
                   hipStream_t stream) {
  if (flags & ~(unsigned)(SAGE_IN_BF16 | SAGE_KV_FP4)) return SAGE_ERR_INVALID_ARG;
  const bool fp4 = (flags & SAGE_KV_FP4) != 0;
  const int rc = check_cache(cache, table, max_pages, S, true, fp4);
  if (rc != SAGE_OK) return rc;
  if (N <= 0 || (long long)cache->Hkv * N > (1LL << 30) || (long long)S * cache->Hkv * N * cache->D > kMaxElems / 64)
    return SAGE_ERR_INVALID_ARG;
  if (!k || !v || !pos || !aligned(k, 16) || !aligned(v, 16) || !aligned(pos, 4) || !aligned(counts, 4) || !aligned(weights, 4))
    return SAGE_ERR_INVALID_ARG;
  if (weights && weights_stride < (long long)max_pages * cache->page_size) return SAGE_ERR_INVALID_ARG;
  sage::Append a;
  a.c = cache_of(cache, table, max_pages, S);
  a.k = k; a.v = v; a.pos = pos; a.counts = counts; a.weights = weights; a.wstride = weights_stride; a.N = N;
  a.ks = strides_or(k_strides, cache->Hkv, N, cache->D);
  a.vs = strides_or(v_strides, cache->Hkv, N, cache->D);
  if (!strides_ok(a.ks, 8, kMaxElems) || !strides_ok(a.vs, 8, kMaxElems)) return SAGE_ERR_INVALID_ARG;
  if (fp4) return hip_status(sage::launch_kv_store(a, nullptr, cache->D, (flags & SAGE_IN_BF16) != 0, sage::kCacheFp4, stream));
  return hip_status(sage::launch_kv_append(a, cache->D, (flags & SAGE_IN_BF16) != 0, stream));
}

int sage_kv_append_slots(const sage_kv_cache* cache, const void* k, const void* v, const sage_strides* k_strides,
                         const sage_strides* v_strides, const int64_t* slots, int B, int N, unsigned flags, hipStream_t stream) {
  if (flags & ~(unsigned)(SAGE_IN_BF16 | SAGE_KV_FP4)) return SAGE_ERR_INVALID_ARG;
  const bool fp4 = (flags & SAGE_KV_FP4) != 0;
  const int rc = check_pages(cache, true, fp4);
  if (rc != SAGE_OK) return rc;
  if (B <= 0 || B > kMaxSeqs || N <= 0 || (long long)cache->Hkv * N > (1LL << 30) ||
      (long long)B * cache->Hkv * N * cache->D > kMaxElems / 64)
    return SAGE_ERR_INVALID_ARG;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return SAGE_ERR_INVALID_ARG;
  sage::Append a;
  a.c = cache_of(cache, nullptr, 0, B);
  a.k = k; a.v = v; a.pos = nullptr; a.counts = nullptr; a.weights = nullptr; a.wstride = 0; a.N = N;
  a.ks = strides_or(k_strides, cache->Hkv, N, cache->D);
  a.vs = strides_or(v_strides, cache->Hkv, N, cache->D);
  if (!strides_ok(a.ks, 8, kMaxElems) || !strides_ok(a.vs, 8, kMaxElems)) return SAGE_ERR_INVALID_ARG;
  const int kind = fp4 ? sage::kCacheFp4 : cache->k_scale ? sage::kCacheInt8 : sage::kCache16;
  return hip_status(sage::launch_kv_store(a, slots, cache->D, (flags & SAGE_IN_BF16) != 0, kind, stream));
}

size_t sage_attn_paged_decode_workspace_size(int S, int Hq, int Hkv, int D, int max_pages, int page_size, int with_weights) {
  if (check_heads(Hq, Hkv, D) != SAGE_OK || S <= 0 || S > kMaxSeqs || max_pages <= 0 || page_size <= 0 ||
      (long long)max_pages * page_size > kMaxCapacity)
    return 0;
  return decode_ws(S, Hq, Hkv, D, max_pages * page_size, with_weights != 0).total;
}

int sage_attn_paged_decode(const sage_kv_cache* cache, const void* q, int64_t q_stride_s, int64_t q_stride_h, void* o,
                           float* lse, const int32_t* table, int max_pages, const int32_t* lens, int S, int Hq, int window,
                           int sinks, float* weights, int64_t weights_stride, unsigned flags, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  if (flags & ~(unsigned)(SAGE_IN_BF16 | SAGE_KV_FP4)) return SAGE_ERR_INVALID_ARG;
  const bool fp4 = (flags & SAGE_KV_FP4) != 0;
  int rc = check_cache(cache, table, max_pages, S, false, fp4);
  if (rc != SAGE_OK) return rc;
  rc = check_heads(Hq, cache->Hkv, cache->D);
  if (rc != SAGE_OK) return rc;
  if (window < 1 || sinks < 0) return SAGE_ERR_INVALID_ARG;
  if (!q || !o || !lens || !aligned(q, 16) || !aligned(o, 16) || !aligned(lens, 4) || !aligned(lse, 4) || !aligned(weights, 4))
    return SAGE_ERR_INVALID_ARG;
  if (!strides_ok(Strides{q_stride_s, q_stride_h, 0}, 8, 0)) return SAGE_ERR_INVALID_ARG;
  const int capacity = max_pages * cache->page_size;
  if (weights && weights_stride < capacity) return SAGE_ERR_INVALID_ARG;
  const DecodeWs w = decode_ws(S, Hq, cache->Hkv, cache->D, capacity, weights != nullptr);
  if (w.total > 0) {
    if (!workspace || !aligned(workspace, 256)) return SAGE_ERR_INVALID_ARG;
    if (workspace_bytes < w.total) return SAGE_ERR_WORKSPACE;
  }
  uint8_t* base = static_cast<uint8_t*>(workspace);
  sage::Decode a;
  a.c = cache_of(cache, table, max_pages, S);
  a.q = q; a.q_s = q_stride_s; a.q_h = q_stride_h;
  a.o = o; a.lse = lse; a.lens = lens; a.Hq = Hq;
  a.window = window; a.sinks = sinks;
  clamp_window(capacity, &a.window, &a.sinks);
  a.weights = weights; a.wstride = weights_stride;
  a.nw = fp4 ? sage::decode_fp4_workgroups(S, Hq, cache->Hkv, capacity) : sage::decode_workgroups(S, Hq, cache->Hkv, capacity);
  a.c2 = softmax_c2(cache->D);
  a.per_page = sage::divide_by(cache->page_size);
  a.part = reinterpret_cast<float*>(base + w.part);
  a.before = a.nw > 0 && w.lse2 > w.line ? reinterpret_cast<long long*>(base + w.line) : nullptr;
  a.lse2 = weights ? reinterpret_cast<float*>(base + w.lse2) : nullptr;
  a.scores = weights ? reinterpret_cast<float*>(base + w.scores) : nullptr;
  a.score_stride = w.score_stride;
  if (fp4) return hip_status(sage::launch_paged_decode_fp4(a, cache->D, (flags & SAGE_IN_BF16) != 0, stream));
  return hip_status(sage::launch_paged_decode(a, cache->D, (flags & SAGE_IN_BF16) != 0, stream));
}

size_t sage_kv_evict_workspace_size(int S, int Hkv, int max_pages, int page_size) {
  if (S <= 0 || S > kMaxSeqs || Hkv <= 0 || Hkv > kMaxHeads || max_pages <= 0 || page_size <= 0 ||
      (long long)max_pages * page_size > kMaxCapacity)
    return 0;
  return up256(sage::evict_hist_ints(S, Hkv, max_pages * page_size) * sizeof(int));
}

int sage_kv_evict(const sage_kv_cache* cache, const int32_t* table, int max_pages, const int32_t* lens, const float* weights,
                  int64_t weights_stride, const int32_t* new_table, int new_max_pages, int budget, int keep_first,
                  int keep_last, int32_t* new_lens, float* new_weights, int32_t* kept, int S, void* workspace,
                  size_t workspace_bytes, hipStream_t stream) {
  return evict(cache, table, max_pages, lens, weights, weights_stride, new_table, new_max_pages, budget, keep_first, keep_last,
               new_lens, new_weights, kept, S, workspace, workspace_bytes, false, stream);
}

int sage_kv_evict_fp4(const sage_kv_cache* cache, const int32_t* table, int max_pages, const int32_t* lens, const float* weights,
                      int64_t weights_stride, const int32_t* new_table, int new_max_pages, int budget, int keep_first,
                      int keep_last, int32_t* new_lens, float* new_weights, int32_t* kept, int S, void* workspace,
                      size_t workspace_bytes, hipStream_t stream) {
  return evict(cache, table, max_pages, lens, weights, weights_stride, new_table, new_max_pages, budget, keep_first, keep_last,
               new_lens, new_weights, kept, S, workspace, workspace_bytes, true, stream);
}

int sage_qk_norm_rope_fwd(const void* q, const void* k, const float* q_weight, const float* k_weight, const float* inv_freq,
                          int rotary, const int32_t* pos, int pos_per_token, const int32_t* lens, void* zq, void* zk, int B,
                          int Hq, int Hkv, int N, int D, float eps, unsigned flags, const sage_strides* q_strides,
                          const sage_strides* k_strides, const sage_strides* zq_strides, const sage_strides* zk_strides,
                          hipStream_t stream) {
  sage::NormRope a{};
  int rc = check_norm_rope(a, q, k, q_weight, k_weight, inv_freq, rotary, pos, pos_per_token, lens, B, Hq, Hkv, N, D, eps, flags,
                           q_strides, k_strides);
  if (rc == SAGE_OK) rc = check_norm_rope_out(a, zq, zk, D, zq_strides, zk_strides);
  if (rc != SAGE_OK) return rc;
  if (!norm_rope_apart(a, D)) return SAGE_ERR_INVALID_ARG;
  return hip_status(sage::launch_norm_rope(a, D, (flags & SAGE_IN_BF16) != 0, (flags & SAGE_ROPE_PAIRS) != 0, false, stream));
}

size_t sage_qk_norm_rope_bwd_workspace_size(int B, int Hq, int Hkv, int N, int D) {
  if (check_heads(Hq, Hkv, D) != SAGE_OK || B <= 0 || N <= 0 || (long long)B * N > (1LL << 30)) return 0;
  return up256((size_t)sage::norm_rope_bwd_blocks((long long)B * N, Hq, Hkv, D) * 2 * D * sizeof(float));
}

int sage_qk_norm_rope_bwd(const void* q, const void* k, const float* q_weight, const float* k_weight, const float* inv_freq,
                          int rotary, const int32_t* pos, int pos_per_token, const int32_t* lens, const void* dzq, const void* dzk,
                          void* dq, void* dk, float* dq_weight, float* dk_weight, int B, int Hq, int Hkv, int N, int D, float eps,
                          unsigned flags, const sage_strides* q_strides, const sage_strides* k_strides,
                          const sage_strides* dzq_strides, const sage_strides* dzk_strides, const sage_strides* dq_strides,
                          const sage_strides* dk_strides, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  sage::NormRope a{};
  int rc = check_norm_rope(a, q, k, q_weight, k_weight, inv_freq, rotary, pos, pos_per_token, lens, B, Hq, Hkv, N, D, eps, flags,
                           q_strides, k_strides);
  if (rc == SAGE_OK) rc = check_norm_rope_out(a, dq, dk, D, dq_strides, dk_strides);
  if (rc != SAGE_OK) return rc;
  if (!dzq || !dzk || !aligned(dzq, 16) || !aligned(dzk, 16) || !aligned(dq_weight, 4) || !aligned(dk_weight, 4))
    return SAGE_ERR_INVALID_ARG;
  a.gq = dzq; a.gk = dzk; a.dwq = dq_weight; a.dwk = dk_weight;
  a.gqs = strides_or(dzq_strides, Hq, N, D); a.gks = strides_or(dzk_strides, Hkv, N, D);
  for (const Strides& s : {a.gqs, a.gks})
    if (!strides_ok(s, 8, kMaxElems)) return SAGE_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256)) return SAGE_ERR_INVALID_ARG;
  if (workspace_bytes < sage_qk_norm_rope_bwd_workspace_size(B, Hq, Hkv, N, D)) return SAGE_ERR_WORKSPACE;
  if (!norm_rope_apart(a, D) || (dq_weight && dq_weight == dk_weight)) return SAGE_ERR_INVALID_ARG;
  a.part = static_cast<float*>(workspace);
  return hip_status(sage::launch_norm_rope(a, D, (flags & SAGE_IN_BF16) != 0, (flags & SAGE_ROPE_PAIRS) != 0, true, stream));
}

int sage_kv_plan(int32_t* table, int max_pages, int32_t* lens, const int32_t* counts, int32_t* free_pages, int free_capacity,
                 int32_t* n_free, int page_size, int32_t* granted, int32_t* starts, int32_t* pos, int64_t* slots, int max_tokens,
                 int S, hipStream_t stream) {
  if (S <= 0 || S > kMaxSeqs || max_pages <= 0 || page_size <= 0 || (long long)max_pages * page_size > kMaxCapacity)
    return SAGE_ERR_INVALID_ARG;
  if (free_capacity <= 0 || max_tokens <= 0 || max_tokens > kMaxCapacity) return SAGE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)table, (const void*)lens, (const void*)counts, (const void*)free_pages, (const void*)n_free,
                        (const void*)granted, (const void*)starts, (const void*)pos})
    if (!p || !aligned(p, 4)) return SAGE_ERR_INVALID_ARG;
  if (!slots || !aligned(slots, 8)) return SAGE_ERR_INVALID_ARG;
  if (counts == lens || counts == granted) return SAGE_ERR_INVALID_ARG;
  sage::Plan a;
  a.table = table; a.lens = lens; a.free_pages = free_pages; a.n_free = n_free; a.counts = counts;
  a.granted = granted; a.starts = starts; a.pos = pos; a.slots = slots;
  a.S = S; a.max_pages = max_pages; a.page_size = page_size; a.free_capacity = free_capacity; a.max_tokens = max_tokens;
  return hip_status(sage::launch_kv_plan(a, stream));
}

}  // extern "C"
