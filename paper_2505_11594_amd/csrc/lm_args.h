// Arguments of the window attention, paged cache and one-token attention
// launchers, as the C entry points fill them in after their checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "window.h"

namespace sage {

struct Strides { long long b, h, n; };   // in elements; channels are contiguous

struct WindowFwd {
  const void *q, *k, *v;
  void* o;
  float* lse;              // may be null
  const int32_t* lens;     // may be null: every sequence has N tokens
  int B, Hq, Hkv, N, window, sinks;
  Strides qs, ks, vs, os;
  float c2;                // log2(e) / sqrt(D)
};
hipError_t launch_window_fwd(const WindowFwd& a, int D, bool bf16, hipStream_t st);

struct WindowBwd {
  const void *q, *k, *v, *o, *dout;
  const float* lse;
  const int32_t* lens;     // may be null
  void *dq, *dk, *dv;      // contiguous
  int B, Hq, Hkv, N, window, sinks;
  int chunks, mchunks, mshare;           // of the sinks' query tiles, of the other keys', and tiles in one of these
  Strides qs, ks, vs, os, gs;            // gs: dout
  float c2, rsd;           // rsd = 1 / sqrt(D)
  float *lb, *delta, *norms, *scales, *part, *mpart;   // workspace
};
int window_bwd_chunks(int B, int Hq, int Hkv, int N, int sinks);
int window_bwd_share(int B, int Hq, int Hkv, int N, int window, int* chunks);
size_t window_bwd_mpart_floats(int B, int Hkv, int N, int D, int chunks);
size_t window_bwd_row_floats(int B, int Hq, int N);
size_t window_bwd_norm_floats(int B, int Hq, int Hkv, int N);
size_t window_bwd_part_floats(int B, int Hq, int Hkv, int N, int D, int sinks);
hipError_t launch_window_bwd(const WindowBwd& a, int D, bool bf16, hipStream_t st);

// A paged cache: pages of page_size tokens, strides in elements; int8 codes with
// one fp32 scale per token and head ([pages, Hkv, page_size], contiguous), 16-bit, or
// MXFP4: strides in bytes, scales are bytes [pages, Hkv, page_size, D / 32].
struct Cache {
  const void *k, *v;
  const float *k_scale, *v_scale;        // null for a 16-bit cache
  Strides ks, vs;                        // b: pages
  int pages, page_size, Hkv;
  const int32_t* table;                  // [S, max_pages]
  int S, max_pages;
};

struct Append {
  Cache c;
  const void *k, *v;                     // [S, Hkv, N, D]
  Strides ks, vs;
  const int32_t *pos, *counts;           // counts may be null
  float* weights;                        // may be null; [S, Hkv, wstride]
  long long wstride;
  int N;
};
hipError_t launch_kv_append(const Append& a, int D, bool bf16, hipStream_t st);
// Every kind of cache, by tables and positions or by slots (int64 [S, N] or null).
enum { kCache16 = 0, kCacheInt8 = 1, kCacheFp4 = 2 };
hipError_t launch_kv_store(const Append& a, const int64_t* slots, int D, bool bf16, int kind, hipStream_t st);

struct Decode {
  Cache c;
  const void* q;                         // [S, Hq, D]
  long long q_s, q_h;
  void* o;                               // [S, Hq, D] contiguous
  float* lse;                            // [S, Hq] or null
  float* weights;                        // [S, Hkv, wstride] or null
  long long wstride;
  const int32_t* lens;
  int Hq, window, sinks, nw;             // nw: workgroups that share the batch's steps (0: one per sequence)
  float c2;
  Divide per_page;                       // by the page size (4-bit caches)
  float* part;                           // per (workgroup, end, head): D sums, then (log2 maximum, sum)
  long long* before;                     // steps before each of more than 64 sequences, or null
  float *lse2, *scores;                  // for weights: [S, Hq], [S, Hq, score_stride]
  long long score_stride;
};
int decode_workgroups(int S, int Hq, int Hkv, int capacity);
size_t decode_line_longs(int S, int Hq, int Hkv, int capacity);
size_t decode_part_floats(int S, int Hq, int Hkv, int D, int capacity);
hipError_t launch_paged_decode(const Decode& a, int D, bool bf16, hipStream_t st);
hipError_t launch_add_weights(const Decode& a, hipStream_t st);
int decode_fp4_workgroups(int S, int Hq, int Hkv, int capacity);
hipError_t launch_paged_decode_fp4(const Decode& a, int D, bool bf16, hipStream_t st);

struct Evict {
  Cache c;
  const int32_t *lens, *new_table;
  const float* weights;
  float* new_weights;
  int32_t *new_lens, *kept;
  long long wstride, new_wstride;
  int new_max_pages, budget, keep_first, keep_last;
  int* hist;                             // workspace; chunks and chunk are the launcher's
  int chunks, chunk;
};
size_t evict_hist_ints(int S, int Hkv, int capacity);
hipError_t launch_kv_evict(const Evict& a, int D, bool fp4, hipStream_t st);

// Norms of queries and keys with their rotation; zq, zk are dq, dk in the backward.
struct NormRope {
  const void *q, *k, *gq, *gk;           // gq, gk: gradients of the outputs
  void *zq, *zk;
  const float *wq, *wk, *freq;           // wq, wk may be null; freq [R / 2]
  const int32_t *pos, *lens;             // may be null
  int B, Hq, Hkv, N, R, pos_each;        // pos [B, N] if pos_each, else [B]: the first token's
  float eps;
  Strides qs, ks, zqs, zks, gqs, gks;
  int split;                             // waves that share a token (the launcher's)
  float *part, *dwq, *dwk;
};
int norm_rope_bwd_blocks(long long tokens, int Hq, int Hkv, int D);
hipError_t launch_norm_rope(const NormRope& a, int D, bool bf16, bool pairs, bool bwd, hipStream_t st);

// Tables and slots of a batch of requests.
struct Plan {
  int32_t *table, *lens, *free_pages, *n_free;       // in and out
  const int32_t* counts;
  int32_t *granted, *starts, *pos;
  int64_t* slots;
  int S, max_pages, page_size, free_capacity, max_tokens;
};
hipError_t launch_kv_plan(const Plan& a, hipStream_t st);

}  // namespace sage
