"""The 64-bit gradients that the GPU tests compare with (_lm.py): against automatic
differentiation and against slopes of the definition; and mistakes planted in them are found (CPU)."""
import math

import pytest

import _lm
import _slopes

CASES = [
    # B, Hq, Hkv, N, D, window, sinks, lens
    (1, 1, 1, 1, 64, None, 0, None),
    (1, 2, 1, 33, 64, 7, 1, None),
    (2, 4, 2, 40, 128, None, 0, [40, 17]),
    (1, 3, 1, 130, 64, 32, 4, None),
    (2, 2, 2, 70, 64, 20, 30, [70, 0]),
    (1, 2, 2, 150, 128, 1, 0, None),
]


def inputs(case):
    import torch
    B, Hq, Hkv, N, D = case[:5]
    g = torch.Generator().manual_seed(N + D)
    r = lambda h: torch.randn((B, h, N, D), generator=g, dtype=torch.float64)
    return [r(Hq), r(Hkv) + torch.randn((B, Hkv, 1, D), generator=g, dtype=torch.float64), r(Hkv)], r(Hq)


def reference(tensors, dout, window, sinks, lens, u=0.0):
    """The gradients and bounds of _lm.py, put together as the GPU tests do."""
    import torch
    q, k, v = tensors
    B, Hq, N, _ = q.shape
    G = Hq // k.shape[1]
    want, bound = ([torch.zeros_like(x) for x in tensors] for _ in range(2))
    for b in range(B):
        n = N if lens is None else lens[b]
        for h in range(Hq):
            r = _lm.window_attention(q[b, h], k[b, h // G], v[b, h // G], window, sinks, n, dout[b, h], u)
            for i, (x, hh) in enumerate((("dq", h), ("dk", h // G), ("dv", h // G))):
                want[i][b, hh] += r[x]
                bound[i][b, hh] += r["e" + x]
    return want, bound


def live(dout, lens):
    g = dout.clone()
    for b, n in enumerate(lens or []):
        g[b, :, n:] = 0
    return g


@pytest.mark.parametrize("case", CASES)
def test_reference_gradients_are_those_of_automatic_differentiation(case):
    window, sinks, lens = case[5:]
    tensors, dout = inputs(case)
    want, _ = reference(tensors, dout, window, sinks, lens)
    t = [x.clone().requires_grad_(True) for x in tensors]
    (_slopes.outputs(*t, window, sinks, lens) * dout).sum().backward()
    for x, w in zip(t, want):
        scale = float(w.abs().max())
        assert float((x.grad - w).abs().max()) <= 1e-12 * case[3] * max(scale, 1e-3)   # N-term sums in 64 bits


@pytest.mark.parametrize("case", CASES[1:])
def test_reference_gradients_are_slopes_and_mistakes_are_not(case):
    import torch
    window, sinks, lens = case[5:]
    tensors, dout = inputs(case)
    zero = [torch.zeros_like(x) for x in tensors]
    want, bound = reference(tensors, dout, window, sinks, lens, u=2.0 ** -8)
    ratios, sizes = _slopes.slopes_agree(tensors, live(dout, lens), want, want, zero, window, sinks, lens)
    alone = window == 1                                  # dQ and dK of a query that sees one key are 0
    assert ratios[2] <= 1 and (alone or max(ratios) <= 1), ratios
    # the kernels' bounds leave less than half of a slope (bf16's here), so that zero does not pass
    got, sizes = _slopes.slopes_agree(tensors, live(dout, lens), zero, want, bound, window, sinks, lens)
    for i in range(2 if alone else 0, 3):
        assert sizes[i] < 0.5 and got[i] > 1.9, (i, sizes, got)
    if alone:
        return
    # delta left out, the softmax scale left out, one query head of a group left out
    q, k, v = tensors
    G = q.shape[1] // k.shape[1]
    wrong = [torch.zeros_like(x) for x in tensors]
    for b in range(q.shape[0]):
        n = q.shape[2] if lens is None else lens[b]
        for h in range(q.shape[1]):
            r = _lm.window_attention(q[b, h], k[b, h // G], v[b, h // G], window, sinks, n)
            ds = r["p"] * (live(dout, lens)[b, h] @ v[b, h // G].T)
            wrong[0][b, h] = ds @ k[b, h // G] / math.sqrt(q.shape[3])
            wrong[1][b, h // G] += ds.T @ q[b, h] / math.sqrt(q.shape[3])
    agree = lambda g: _slopes.slopes_agree(tensors, live(dout, lens), g, want, bound, window, sinks, lens)[0]
    assert agree(wrong[:2] + want[2:])[0] > 1            # (along dK it is within the bounds for some of these)
    assert max(agree([x * math.sqrt(q.shape[3]) for x in want[:2]] + want[2:])[:2]) > 1
    if G > 1:
        only = [torch.zeros_like(x) for x in tensors]
        for b in range(q.shape[0]):
            n = q.shape[2] if lens is None else lens[b]
            for h in range(0, q.shape[1], G):
                r = _lm.window_attention(q[b, h], k[b, h // G], v[b, h // G], window, sinks, n, dout[b, h])
                only[1][b, h // G], only[2][b, h // G] = r["dk"], r["dv"]
        got = agree([want[0], only[1], only[2]])
        assert got[1] > 1 and got[2] > 1, got
