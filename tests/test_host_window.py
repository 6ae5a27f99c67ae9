"""The integer code of the window and cache kernels, run on the host: the key
tiles of csrc/window.h cover what a query sees, each tile once, and the forward
kernel's own skip and mask conditions keep exactly the visible keys."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11594_amd", "csrc")

MAIN = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include "window.h"
using namespace sage;
using std::min;
static long long bad = 0, seen = 0;
static bool sees(int i, int j, int n, int window, int sinks) {
  return j <= i && j < n && ((long long)j > (long long)i - window || j < sinks);
}
static void lists(int lo, int hi, int sinks, int T) {
  const TileList t = tile_list(lo, hi, sinks, T);
  int last = -1;
  for (int i = 0; i < t.count; ++i) {
    if (t.tile(i) <= last || t.tile(i) * T >= hi) ++bad;
    last = t.tile(i);
  }
  for (int j = 0; j < hi; ++j)
    if (j < sinks || j >= lo) {
      bool in = false;
      for (int i = 0; i < t.count; ++i) in |= t.tile(i) == j / T;
      bad += !in;
      ++seen;
    }
}
// the forward kernel's tile loop for the queries of one wave
static void forward(int n, int N, int W, int sinks) {
  constexpr int WK = 64, WW = 4;
  for (int q0 = 0; q0 < N && q0 < n; q0 += 32 * WW)
    for (int wave = 0; wave < WW; ++wave)
      for (int col = 0; col < 32; ++col) {
        const int qw = q0 + wave * 32, qi = qw + col;
        if (qi >= n) continue;
        @TILES@
        static unsigned char got[4096];
        for (int j = 0; j < n; ++j) got[j] = 0;
        for (int j = 0; j < tl.count; ++j) {
          @HALVES@
          const auto piece = [&](int NS, int kb) {
            bool masked = false;
            @COND@ masked = true;
            for (int hi = 0; hi < 2; ++hi)
              for (int t = 0; t < NS; ++t)
                for (int e = 0; e < 16; ++e) {
                  @BASE@
                  const int c = 32 * t + 8 * (e >> 2) + (e & 3);
                  uint32_t keep_ = ~0u;
                  if (masked) { @KEEP@ keep_ = keep; }
                  if (keep_) { if (base + c >= n) ++bad; else ++got[base + c]; }
                }
          };
          if (hide0 && hide1) continue;
          if (!hide0 && !hide1) piece(2, kb);
          else piece(1, hide0 ? kb + 32 : kb);
        }
        for (int j = 0; j < n; ++j) { bad += got[j] != (sees(qi, j, n, W, sinks) ? 1 : 0); ++seen; }
      }
}
int main() {
  for (int T : {32, 64})
    for (int hi : {0, 1, 31, 32, 33, 64, 100, 129, 300})
      for (int lo = -40; lo <= hi; lo += 7)
        for (int sinks : {0, 1, 4, 31, 32, 33, 64, 70, 200, 400}) lists(lo, hi, sinks, T);
  for (int n : {0, 1, 5, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 333, 700})
    for (int W : {1, 2, 31, 32, 33, 63, 64, 65, 95, 100, 127, 128, 129, 159, 256, 1000})
      for (int sinks : {0, 1, 4, 33, 64, 70, 130, 400}) {
        int w = W < 700 ? W : 700, s = w >= 700 ? 0 : sinks;
        forward(n, 700, w, s);
      }
  // one new token
  for (int n : {0, 1, 31, 32, 33, 100, 129, 1000})
    for (int W : {1, 7, 32, 100, 1 << 30})
      for (int sinks : {0, 1, 40, 5000}) {
        const TileList t = decode_tiles(n, W, sinks, 32);
        for (int j = 0; j < n; ++j) {
          bool in = false;
          for (int i = 0; i < t.count; ++i) in |= t.tile(i) == j / 32;
          if (decode_sees(j, n, W, sinks) != sees(n - 1, j, n, W, sinks)) ++bad;
          if (sees(n - 1, j, n, W, sinks) && !in) ++bad;
          ++seen;
        }
      }
  for (unsigned groups : {1u, 2u, 3u, 7u, 8u, 16u, 24u, 96u, 100u})       // every piece once, runs on one XCD
    for (unsigned per : {1u, 2u, 5u, 10u, 257u}) {
      static int who[1 << 15];
      const unsigned total = groups * per;
      for (unsigned i = 0; i < total; ++i) who[i] = -1;
      for (unsigned b = 0; b < total; ++b) {
        const unsigned l = xcd_order(b, total, groups);
        if (l >= total || who[l] >= 0) { ++bad; continue; }
        who[l] = (int)(b & 7);
      }
      if (groups % 8 == 0)
        for (unsigned i = 0; i < total; ++i) bad += who[i] != who[i / per * per] || who[i] != (int)(i / per % 8);
    }
  bad += cached_len(-5, 100) != 0 || cached_len(101, 100) != 100 || cached_len(7, 100) != 7;
  bad += page_ok(-1, 4) || page_ok(4, 4) || !page_ok(0, 4) || !page_ok(3, 4) || page_ok(INT32_MIN, 4);
  printf("%lld pairs, %lld wrong\n", seen, bad);
  return bad != 0;
}
"""


def between(src, a, b):
    i = src.index(a)
    return src[i:src.index(b, i) + len(b)]


def program(planted=False):
    src = open(os.path.join(CSRC, "attn_window.hip")).read()
    tiles = between(src, "const int q1 = min(q0 + 32 * WW, n);", "TileList{0, 0, 0};")
    halves = between(src, "const int kb = tl.tile(j) * WK;", "if (hide0 && hide1)")[:-len("if (hide0 && hide1)")]
    cond = between(src, "if (kb + 32 * NS - 1 > qw ||", ") {")[:-1]
    base = between(src, "const int base = kb + 4 * hi,", ";")
    keep = between(src, "const uint32_t keep = ", ";")
    if planted:
        cond = cond.replace("kb <= qw + 31 - W", "kb < qw + 31 - W")
    text = MAIN
    for name, code in (("@TILES@", tiles), ("@HALVES@", halves), ("@COND@", cond), ("@BASE@", base), ("@KEEP@", keep)):
        text = text.replace(name, code)
    return text


def _run(tmp_path, text):
    (tmp_path / "t.cpp").write_text(text)
    exe = str(tmp_path / "t")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I" + CSRC, "-o", exe, str(tmp_path / "t.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    print(r.stdout)
    return r


def test_tiles_and_masks_are_the_visible_keys(tmp_path):
    r = _run(tmp_path, program())
    assert r.returncode == 0, r.stdout


def test_a_mask_condition_that_is_one_off_is_found(tmp_path):
    r = _run(tmp_path, program(planted=True))
    assert r.returncode != 0, r.stdout
