"""Division by multiplication (csrc/window.h), run on the host against the division itself."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11594_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include "window.h"
using namespace sage;
static long long bad = 0, seen = 0;
static void check(const Divide& d, long long n) {
  if (n < 0 || n > 0x7FFFFFFFLL) return;
  bad += d((int)n) != (int)(n / d.by);
  ++seen;
}
static void all(int by) {
  const Divide d = divide_by(by);
  for (long long n = 0; n < 300; ++n) check(d, n);
  for (long long n = 0x7FFFFFFFLL - 300; n <= 0x7FFFFFFFLL; ++n) check(d, n);
  // around multiples, spread over the range
  const long long m = 0x7FFFFFFFLL / by, step = m / 500 + 1;
  for (long long k = 0; k <= m; k += step)
    for (int e = -1; e <= 1; ++e) check(d, k * by + e);
  for (int b = 0; b < 31; ++b)
    for (int e = -1; e <= 1; ++e) check(d, (1LL << b) + e);
}
int main() {
  for (int by = 1; by <= 5000; ++by) all(by);
  for (int b = 12; b <= 30; ++b)
    for (int e = -3; e <= 3; ++e) all((1 << b) + e);
  unsigned x = 12345;
  for (int i = 0; i < 3000; ++i) {
    x = x * 1664525u + 1013904223u;
    all((int)(x >> (1 + x % 20)) | 1);
  }
  all(0x7FFFFFFF);
  std::printf("%lld %lld", bad, seen);
  return 0;
}
"""


def test_division_by_multiplication(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)])
    bad, seen = (int(x) for x in subprocess.check_output([str(exe)]).split())
    assert bad == 0 and seen > 10 ** 6
