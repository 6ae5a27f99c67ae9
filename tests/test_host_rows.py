"""Whether two strided tensors meet (csrc/rows.h), run on the host against every element's address."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11594_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include "rows.h"
using namespace sage;
int main() {
  long long D, x[13];
  for (;;) {
    if (std::scanf("%lld", &D) != 1) return 0;
    for (long long& v : x)
      if (std::scanf("%lld", &v) != 1) return 1;
    const RowSet a((int)D, x[0], x[1], x[2], x[3], x[4], x[5]), b((int)D, x[6], x[7], x[8], x[9], x[10], x[11]);
    int steps = 4096;
    const bool meet = rows_meet(a, 0, b, 0, x[12], &steps);
    std::printf("%d %d\n", (int)meet, steps);
  }
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    src, exe = d / "main.cpp", d / "main"
    src.write_text(MAIN)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)])

    def run(cases):
        """Cases (D, (sb, nb, sh, nh, sn, nn) of a, the same of b, d): answers and the steps that were left."""
        text = "\n".join(" ".join(str(x) for x in (D,) + a + b + (d,)) for D, a, b, d in cases)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def elements(D, t, at):
    sb, nb, sh, nh, sn, nn = t
    return {at + b * sb + h * sh + n * sn + c for b in range(nb) for h in range(nh) for n in range(nn) for c in range(D)}


def test_every_address(meet):
    """Small tensors of any strides (broadcast, overlapping, of one buffer, of two) at any distance."""
    rng = random.Random(1)
    cases = []
    for _ in range(6000):
        D = rng.choice([1, 2, 3, 4])
        size = lambda: rng.choice([1, 2, 2, 3, 4, 5])
        stride = lambda: rng.choice([0, 1, 2, 3, 4, 5, 6, 8, 9, 12, 15, 16, 20, 24, 40, 60, 80])
        a = tuple(x for _ in range(3) for x in (stride(), size()))
        b = tuple(x for _ in range(3) for x in (stride(), size()))
        if rng.random() < 0.5:                           # the same strides, other sizes
            b = tuple(a[i] if i % 2 == 0 else b[i] for i in range(6))
        cases.append((D, a, b, rng.randint(-120, 120)))
    yes = 0
    for (D, a, b, d), (got, left) in zip(cases, meet(cases)):
        want = bool(elements(D, a, 0) & elements(D, b, d))
        assert bool(got) == want and left >= 0, (D, a, b, d)
        yes += want
    assert 1000 < yes < 5000


def test_views_of_large_buffers_take_few_steps(meet):
    """q, k and v of one packed projection, padded and transposed ones, blocks of one workspace: hardly any steps."""
    B, N, H, Hkv, D = 16, 1 << 20, 32, 8, 128
    T = H + 2 * Hkv
    q, k = (N * T * D, B, D, H, T * D, N), (N * T * D, B, D, Hkv, T * D, N)
    cases = [(D, q, k, H * D, 0), (D, q, q, 0, 1), (D, q, k, (H - 1) * D, 1), (D, q, k, -Hkv * D, 0), (D, q, k, -D, 1),
             (D, q, k, (T + H) * D, 0), (D, q, k, -(T - H) * D, 0), (D, q, k, N * T * D * B, 0), (D, q, k, 3 * N * T * D + 5 * T * D + 7, 1)]
    # per sequence first q's rows by token, then z's by head
    b = (2 * N * H * D, B, D, H, H * D, N)
    z = (2 * N * H * D, B, N * D, H, D, N)
    cases += [(D, b, z, N * H * D, 0), (D, b, z, N * H * D - 1, 1), (D, b, z, -N * H * D, 0), (D, z, b, N * H * D, 0), (D, b, z, -N * H * D + 1, 1)]
    # every second row, every fourth of the others
    cases += [(D, (0, 1, 0, 1, 2 * D, N), (0, 1, 0, 1, 2 * D, N), D, 0), (D, (0, 1, 0, 1, 2 * D, N), (0, 1, 0, 1, 2 * D, N), D - 8, 1)]
    # contiguous at q's own address, though q's rows lie apart
    cases += [(D, q, (N * H * D, B, N * D, H, D, N), 0, 1), (D, q, (N * H * D, B, D, H, H * D, N), 0, 1)]
    for (D, a, b, d, want), (got, left) in zip(cases, meet([c[:4] for c in cases])):
        assert got == want and left > 4096 - 200, (a, b, d, left)
