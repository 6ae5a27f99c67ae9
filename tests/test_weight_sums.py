"""The weights' gradients of the norms with rotation, to within the additions that the kernel makes; and that this bound
sees what is missing (on the host, with mistakes in the definition's own sums)."""
import pytest

from paper_2505_11594_amd import binding as bd

import _more_lm as mo
import _weight_sums as ws
from _gpu import torch_dev, say
from test_gpu_more_lm import ROPES

MORE = [
    # more waves than one round of workgroups holds: two to four tokens a wave, in q's and in k's sums
    (1, 16, 16, 13000, 64, 64, False, "bf16", "0", None, False, True),
    (2, 32, 8, 5000, 128, 128, True, "fp16", "each", [5000, 4097], False, True),
    (3, 5, 5, 2731, 128, 64, False, "bf16", "start", None, False, True),
]


def test_additions_of_known_launches():
    assert ws.additions(1, 1, 1, 1, 64) == [1 + 5 + 1 + 6] * 2
    assert ws.additions(1, 32, 8, 8192, 128) == [2 * 8 + 4 + 16 + 6, 2 * 2 + 4 + 16 + 6]
    assert ws.additions(1, 16, 1, 5000, 64) == [2 * 2 + 5 + 16 + 6, 2 + 5 + 16 + 6]


@pytest.mark.parametrize("case", ROPES + MORE)
def test_the_bound_sees_gradients_that_lack_something(case):
    """A gradient of zeros, one of half the size, and one that lacks a row, any of some, are all out of the bound."""
    import torch
    q, k, w, inv, p, live, dq, dk, _ = ws.make(case, "cpu")
    rows_live = lambda H: live.expand(-1, H, -1, -1).reshape(-1)
    for (terms, tol), H in zip(ws.weight_gradients(case, q, k, w, inv, p, live, dq, dk), case[1:3]):
        dw = terms.sum(0)
        outside = lambda x: (x - dw).abs() > tol
        assert float(outside(0 * dw).double().mean()) >= 0.98 and float(outside(dw / 2).double().mean()) >= 0.98
        real = rows_live(H).nonzero()[:, 0]
        for i in {0, len(real) // 3, len(real) // 2, len(real) - 1}:
            assert bool(outside(dw - terms[real[i]]).any()), i
        # whole heads, the last tokens of all heads
        by_head = terms.unflatten(0, (case[0], H, case[3])).sum((0, 2))
        assert all(bool(outside(dw - x).any()) for x in by_head)


@pytest.mark.gpu
@pytest.mark.parametrize("case", ROPES + MORE)
def test_weight_gradients(case):
    import torch
    torch_dev()
    say("weights' gradients %s" % (case,))
    q, k, w, inv, p, live, dq, dk, kw = ws.make(case, "cuda")
    got = bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dq, dk, **kw)[2:]
    torch.cuda.synchronize()
    th = mo.angles(inv, p)[:, None]
    for x, wt, dz, g, (terms, tol) in zip((q, k), w, (dq, dk), got, ws.weight_gradients(case, q, k, w, inv, p, live, dq, dk)):
        dw = terms.sum(0)
        at = float(((g.double() - dw).abs() / tol).max())
        say("  dw at %.3f of its bound" % at)
        assert at <= 1
        # against differences: the loss sum(z dz) is linear in the weights
        x64, dz64 = torch.where(live, x.double(), 0.0), torch.where(live, dz.double(), 0.0)
        loss = lambda ww: float((mo.norm_rope(x64, ww, th, case[6], 1e-5, live)[1] * dz64).sum())
        slope = (loss(wt.double() + dw) - loss(wt.double() - dw)) / 2
        assert abs(float((g.double() * dw).sum()) - slope) <= float((tol * dw.abs()).sum()) + 1e-9 * abs(slope) + 1e-9
