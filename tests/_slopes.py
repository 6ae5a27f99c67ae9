"""Gradients of the window attention checked against slopes of its definition, without the
formulas of _lm.py: along one tensor's gradient at a time, so that the slope is the
gradient's own square and a gradient that is zero, or lacks a term, cannot pass."""
import math


def outputs(q, k, v, window, sinks, lens):
    """O of a batch with grouped heads in 64 bits, 0 behind a sequence's end.  q [B, Hq, N, D],
    k, v [B, Hkv, N, D]."""
    import torch
    B, Hq, N, D = q.shape
    i, j = torch.arange(N, device=q.device)[:, None], torch.arange(N, device=q.device)[None, :]
    hidden = (j > i) | (False if window is None else (i - j >= window) & (j >= sinks))
    n = torch.full((B,), N, device=q.device) if lens is None else torch.tensor(lens, device=q.device).clamp(0, N)
    live = (torch.arange(N, device=q.device) < n[:, None])[:, None, :, None]
    k, v = (x.repeat_interleave(Hq // k.shape[1], 1) for x in (k, v))
    x = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    # (a key behind the end is in the future of every live query)
    return torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v * live


def slope(tensors, which, d, dout, window, sinks, lens):
    """d/dt of sum(O dO) with tensor `which` moved by t d: central differences at t and t / 2, of
    which the terms of second order cancel.  The rest is of order t^4 = 1e-12 relative."""
    def loss(t):
        x = list(tensors)
        x[which] = x[which] + t * d
        return float((outputs(*x, window, sinks, lens) * dout).sum())

    t = 1e-3 / max(1e-300, float(d.square().mean().sqrt()))
    near, far = ((loss(h) - loss(-h)) / (2 * h) for h in (t / 2, t))
    return (4 * near - far) / 3


def slopes_agree(tensors, dout, grads, want, bound, window, sinks, lens):
    """For each tensor: |<grad, d> - slope along d| <= sum(bound |d|) + 1e-6 |slope| for d = want.
    Returns the three ratios, and how large the tolerances are next to their slopes."""
    ratios, sizes = [], []
    for i, (g, d, t) in enumerate(zip(grads, want, bound)):
        s = slope(tensors, i, d, dout, window, sinks, lens)
        tol = float((t * d.abs()).sum()) + 1e-6 * abs(s) + 1e-12
        ratios.append(abs(float((g.double() * d).sum()) - s) / tol)
        sizes.append(tol / max(1e-300, abs(s)))
    return ratios, sizes
