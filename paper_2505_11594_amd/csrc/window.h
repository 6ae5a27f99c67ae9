// Which keys a query sees under a causal sliding window with sinks, and the key
// tiles that hold them; the pages of a cached sequence; the shares of a split
// over many sequences.  Plain integer code, for the kernels and for the host.
//
// Query i of a sequence of n tokens sees key j iff
//   j <= i  and  j < n  and  (j > i - window  or  j < sinks).
// With window >= n the sinks add nothing.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define SAGE_HD __host__ __device__ __forceinline__
#else
#define SAGE_HD inline
#endif

namespace sage {

SAGE_HD int imin(int a, int b) { return a < b ? a : b; }
SAGE_HD int imax(int a, int b) { return a > b ? a : b; }
SAGE_HD int cdiv(int a, int b) { return (a + b - 1) / b; }

// The tiles of T keys that hold the keys [0, sinks) and [lo, hi): first the
// tiles [0, n1), then those from t0 on; `count` in all, each once.
struct TileList {
  int n1, t0, count;
  SAGE_HD int tile(int i) const { return i < n1 ? i : t0 + (i - n1); }
};
SAGE_HD TileList tile_list(int lo, int hi, int sinks, int T) {
  TileList t;
  if (hi <= 0) { t.n1 = t.t0 = t.count = 0; return t; }
  lo = imax(0, imin(lo, hi));
  t.n1 = cdiv(imin(imin(sinks, lo), hi), T);       // sinks in front of the window
  t.t0 = imax(t.n1, lo / T);
  t.count = t.n1 + imax(0, cdiv(hi, T) - t.t0);
  return t;
}

// A new token's view of its cached sequence of n tokens (itself the last one).
SAGE_HD TileList decode_tiles(int n, int window, int sinks, int T) { return tile_list(n - window, n, sinks, T); }
SAGE_HD bool decode_sees(int j, int n, int window, int sinks) { return j < n && (j >= n - window || j < sinks); }

// Length of a cached sequence as the kernels take it: what its pages can hold.
SAGE_HD int cached_len(int n, int capacity) { return imax(0, imin(n, capacity)); }

// A page id is used only if the cache has that page.
SAGE_HD bool page_ok(int id, int pages) { return (unsigned)id < (unsigned)pages; }

// Which of `total` pieces of work, `groups` equal runs that share keys, a block takes.
// Blocks go to the 8 XCDs in turn; every run stays on one (its keys in one L2).  Runs
// are dealt out in turn where 8 divides them, so that sequences of differing lengths
// spread over the XCDs; else each XCD takes an equal part of the line.
SAGE_HD unsigned xcd_order(unsigned block, unsigned total, unsigned groups) {
  const unsigned x = block & 7, i = block >> 3;
  if (groups % 8 == 0) {
    const unsigned per = total / groups, run = i / per;
    return (run * 8 + x) * per + (i - run * per);
  }
  const unsigned more = total & 7;
  return x * (total >> 3) + (x < more ? x : more) + i;
}

}  // namespace sage
