// C ABI of the window attention, the paged cache and one-token attention over it.
// Argument checks run on the host before any HIP call; kernels are enqueued on the
// caller's stream; nothing is allocated.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "lm_args.h"
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
int check_cache(const sage_kv_cache* c, const int32_t* table, int max_pages, int S, bool written) {
  if (!c || !c->k || !c->v || !table || !aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(table, 4)) return SAGE_ERR_INVALID_ARG;
  if (!c->k_scale != !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return SAGE_ERR_INVALID_ARG;
  if (c->pages <= 0 || c->page_size <= 0 || max_pages <= 0 || S <= 0 || S > kMaxSeqs) return SAGE_ERR_INVALID_ARG;
  if ((long long)max_pages * c->page_size > kMaxCapacity) return SAGE_ERR_INVALID_ARG;
  if (check_heads(c->Hkv, c->Hkv, c->D) != SAGE_OK) return SAGE_ERR_INVALID_ARG;
  const int per = c->k_scale ? 16 : 8;
  for (const sage_strides* s : {&c->k_strides, &c->v_strides}) {
    const Strides x{s->b, s->h, s->n};
    if (!strides_ok(x, per, kMaxElems)) return SAGE_ERR_INVALID_ARG;
    if (written && !distinct_rows(x, c->pages, c->Hkv, c->page_size, c->D)) return SAGE_ERR_INVALID_ARG;
  }
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
  if (flags & ~(unsigned)SAGE_IN_BF16) return SAGE_ERR_INVALID_ARG;
  const int rc = check_cache(cache, table, max_pages, S, true);
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
  return hip_status(sage::launch_kv_append(a, cache->D, (flags & SAGE_IN_BF16) != 0, stream));
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
  if (flags & ~(unsigned)SAGE_IN_BF16) return SAGE_ERR_INVALID_ARG;
  int rc = check_cache(cache, table, max_pages, S, false);
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
  a.nw = sage::decode_workgroups(S, Hq, cache->Hkv, capacity);
  a.c2 = softmax_c2(cache->D);
  a.part = reinterpret_cast<float*>(base + w.part);
  a.before = w.lse2 > w.line ? reinterpret_cast<long long*>(base + w.line) : nullptr;
  a.lse2 = weights ? reinterpret_cast<float*>(base + w.lse2) : nullptr;
  a.scores = weights ? reinterpret_cast<float*>(base + w.scores) : nullptr;
  a.score_stride = w.score_stride;
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
  const int rc = check_cache(cache, table, max_pages, S, true);
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
  return hip_status(sage::launch_kv_evict(a, cache->D, stream));
}

}  // extern "C"
