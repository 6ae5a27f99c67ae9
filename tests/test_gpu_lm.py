"""GPU checks of window attention, the paged cache, one-token attention and
eviction against their definitions in 64 bits (_lm.py, which derives the bounds)."""
import math

import numpy as np
import pytest

from paper_2505_11594_amd import binding as bd

import _lm
from _gpu import torch_dev, say

pytestmark = pytest.mark.gpu

DT = {"bf16": "bfloat16", "fp16": "float16"}


def gen(seed):
    torch = torch_dev()
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda")


def qkv(seed, B, Hq, Hkv, N, D, dtype):
    import torch
    g = gen(seed)
    dt = getattr(torch, DT[dtype])
    k = randn(g, B, Hkv, N, D) + randn(g, B, Hkv, 1, D)
    return randn(g, B, Hq, N, D).to(dt), k.to(dt), randn(g, B, Hkv, N, D).to(dt)


def check_window(q, k, v, o, lse, window, sinks, lens, label):
    import torch
    B, Hq, N, D = q.shape
    G, u = Hq // k.shape[1], _lm.unit(q.dtype)
    worst = [0.0, 0.0]
    for b in range(B):
        n = N if lens is None else max(0, min(N, int(lens[b])))
        for h in range(Hq):
            r = _lm.window_attention(q[b, h].double(), k[b, h // G].double(), v[b, h // G].double(), window, sinks, n)
            t = _lm.o_bound(r, n, u)
            worst[0] = max(worst[0], float(((o[b, h].double() - r["o"]).abs() / t)[:n].max()) if n else 0.0)
            assert bool((o[b, h, n:] == 0).all()), label
            if lse is not None:
                assert bool((lse[b, h, n:] == -math.inf).all()), label
                if n:
                    worst[1] = max(worst[1], float(((lse[b, h].double() - r["lse"]).abs() / _lm.lse_bound(r, n))[:n].max()))
    say("%s: O at %.3f of its bound, L at %.3f" % (label, *worst))
    assert worst[0] <= 1 and worst[1] <= 1, label


WINDOWS = [
    # B, Hq, Hkv, N, D, dtype, window, sinks, lens
    (1, 1, 1, 1, 64, "bf16", None, 0, None),
    (1, 2, 1, 1, 128, "fp16", 1, 0, None),
    (2, 4, 2, 64, 128, "bf16", 1, 0, None),
    (1, 4, 4, 65, 64, "fp16", 7, 1, None),
    (1, 6, 2, 127, 128, "bf16", 32, 4, None),
    (2, 2, 1, 129, 64, "bf16", 33, 0, None),
    (1, 8, 1, 300, 128, "fp16", 64, 64, None),
    (1, 2, 2, 300, 128, "bf16", 100, 70, None),
    (1, 2, 2, 257, 64, "fp16", None, 5, None),
    (1, 3, 3, 1000, 128, "bf16", 128, 130, None),
    (1, 2, 1, 1000, 64, "bf16", 500, 16, None),
    (1, 2, 2, 700, 128, "fp16", 1000, 3, None),
    (1, 2, 2, 700, 128, "bf16", 699, 0, None),
    (1, 2, 2, 700, 64, "bf16", 95, 2, None),
    (4, 4, 2, 200, 64, "fp16", 50, 4, [200, 0, 1, 129]),
    (5, 2, 1, 300, 128, "bf16", None, 0, [300, 64, -7, 255, 1000]),
    (3, 7, 1, 513, 128, "bf16", 257, 1, [513, 512, 128]),
    # more than a workgroup per CU: one group of waves each (the others run two)
    (2, 32, 8, 600, 128, "bf16", 200, 4, [600, 333]),
    (2, 32, 16, 600, 64, "fp16", 200, 40, None),
    (1, 64, 4, 650, 64, "bf16", None, 0, None),
    (1, 64, 32, 550, 128, "fp16", None, 0, None),
    # enough key blocks of like length that none is cut into chunks in the backward
    (4, 32, 32, 512, 64, "bf16", 64, 0, None),
    (4, 32, 32, 512, 128, "fp16", 64, 4, [512, 511, 300, 0]),
]


@pytest.mark.parametrize("case", WINDOWS)
def test_window_forward(case):
    import torch
    B, Hq, Hkv, N, D, dtype, window, sinks, lens = case
    q, k, v = qkv(11 + N + D, B, Hq, Hkv, N, D, dtype)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=window, sinks=sinks, lens=ln)
    torch.cuda.synchronize()
    check_window(q, k, v, o, lse, window, sinks, lens, "window %s" % (case,))


def check_grads(q, k, v, dout, grads, window, sinks, lens, label):
    """dQ, dK, dV within their bounds; returns the references and bounds for other uses."""
    import torch
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    G, u = Hq // Hkv, _lm.unit(q.dtype)
    want = [torch.zeros(x.shape, dtype=torch.float64, device=x.device) for x in (q, k, v)]
    bound = [torch.zeros_like(x) for x in want]
    for b in range(B):
        n = N if lens is None else max(0, min(N, int(lens[b])))
        for h in range(Hq):
            r = _lm.window_attention(q[b, h].double(), k[b, h // G].double(), v[b, h // G].double(), window, sinks, n,
                                     dout[b, h].double(), u)
            for i, (x, hh) in enumerate((("dq", h), ("dk", h // G), ("dv", h // G))):
                want[i][b, hh] += r[x]
                bound[i][b, hh] += r["e" + x]
    worst = []
    for x, w, t in zip(grads, want, bound):
        t = t + u * (w.abs() + t) + torch.finfo(x.dtype).smallest_normal * 2.0 ** -10
        worst.append(float(((x.double() - w).abs() / t).max()))
        for b in range(B):
            n = N if lens is None else max(0, min(N, int(lens[b])))
            assert bool((x[b, :, n:] == 0).all()), label
    say("%s: dQ at %.3f of its bound, dK %.3f, dV %.3f" % (label, *worst))
    assert max(worst) <= 1, label
    return want, bound


@pytest.mark.parametrize("case", WINDOWS)
def test_window_backward(case):
    import torch
    B, Hq, Hkv, N, D, dtype, window, sinks, lens = case
    q, k, v = qkv(12 + N + D, B, Hq, Hkv, N, D, dtype)
    dout = randn(gen(N), B, Hq, N, D).to(q.dtype)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    say("backward %s" % (case,))
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=window, sinks=sinks, lens=ln)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=window, sinks=sinks, lens=ln)
    torch.cuda.synchronize()
    want, bound = check_grads(q, k, v, dout, grads, window, sinks, lens, "backward %s" % (case,))
    again = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=window, sinks=sinks, lens=ln)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    # against differences of the definition in 64 bits, along one direction
    d = [randn(gen(N + i), *x.shape).double() for i, x in enumerate((q, k, v))]

    def loss(t):
        x, y, z = (a.double() + t * b for a, b in zip((q, k, v), d))
        s = 0.0
        for b in range(B):
            n = N if lens is None else max(0, min(N, int(lens[b])))
            for h in range(Hq):
                kv = h * Hkv // Hq
                s += float((_lm.window_attention(x[b, h], y[b, kv], z[b, kv], window, sinks, n)["o"] * dout[b, h].double())[:n].sum())
        return s

    t = 1e-4
    slope = (loss(t) - loss(-t)) / (2 * t)
    got = sum(float((g.double() * x).sum()) for g, x in zip(grads, d))
    u = _lm.unit(q.dtype)
    tol = sum(float(((e + u * (w.abs() + e)) * x.abs()).sum()) for e, w, x in zip(bound, want, d))
    # a difference of second order in t, whose third derivative the scores bound loosely; rounding of the losses
    scale = sum(float((w.abs() * x.abs()).sum()) for w, x in zip(want, d))
    assert abs(got - slope) <= tol + 1e-3 * scale + 1e-6, (got, slope, tol)


@pytest.mark.parametrize("dtype,scale", [("fp16", 1e-4), ("fp16", 3e2), ("bf16", 1e-6), ("bf16", 1e6)])
def test_window_backward_small_and_large_gradients(dtype, scale):
    """dO far from 1, its rows of very different size: fp16's dS keeps its precision."""
    import torch
    q, k, v = qkv(60, 1, 4, 2, 333, 64, dtype)
    dout = (randn(gen(61), 1, 4, 333, 64) * scale * torch.exp(randn(gen(62), 1, 4, 333, 1))).to(q.dtype)
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=100, sinks=5)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=100, sinks=5)
    torch.cuda.synchronize()
    check_grads(q, k, v, dout, grads, 100, 5, None, "dO x %g" % scale)
    zero = bd.sage_attn_window_bwd(q, k, v, o, lse, torch.zeros_like(dout), window=100, sinks=5)
    assert all(bool((x == 0).all()) for x in zero)


def test_window_backward_strides_padding_and_buffers():
    """[B, N, H, D] tensors and given buffers: the bits of contiguous copies; what lies behind a
    sequence's end (NaN here) is not read; gradients of broadcast heads add up to the group's."""
    import torch
    B, Hq, Hkv, N, D = 2, 4, 2, 200, 128
    q, k, v = qkv(70, B, Hq, Hkv, N, D, "bf16")
    dout = randn(gen(71), B, Hq, N, D).to(q.dtype)
    lens = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    kw = dict(window=50, sinks=40, lens=lens)
    o, lse = bd.sage_attn_window_fwd(q, k, v, **kw)
    ref = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, **kw)
    tr = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, o, dout)]
    bad = [x.clone() for x in tr]
    for x in bad:
        x[1, :, 77:] = float("nan")
    lb = lse.clone()
    lb[1, :, 77:] = float("nan")
    ws = torch.full((bd.attn_window_bwd_workspace_size(B, Hq, Hkv, N, D, 50, 40),), 255, dtype=torch.uint8, device="cuda")
    out = [torch.full_like(x, 3.0) for x in ref]
    for t, l in ((tr, lse), (bad, lb)):
        got = bd.sage_attn_window_bwd(t[0], t[1], t[2], t[3], l, t[4], workspace=ws, out=out, **kw)
        torch.cuda.synchronize()
        assert all(a is b for a, b in zip(got, out)) and all(torch.equal(a, b) for a, b in zip(got, ref))
        for x in out:
            x.fill_(5.0)
    wide = [x.repeat_interleave(2, 1) for x in (k, v)]
    o2, lse2 = bd.sage_attn_window_fwd(q, *wide, **kw)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    g2 = bd.sage_attn_window_bwd(q, *wide, o, lse, dout, **kw)
    torch.cuda.synchronize()
    assert torch.equal(g2[0], ref[0])
    for a, b in zip(g2[1:], ref[1:]):
        a = a.float().view(B, Hkv, 2, N, D)
        lim = 2.0 ** -8 * (a.abs().sum(2) + b.float().abs()) + 2.0 ** -18 * float(a.abs().max())
        assert bool(((a.sum(2) - b.float()).abs() <= lim).all())


def test_window_training_step_captured():
    """Forward and backward captured into one graph; replayed with new inputs, eager calls between."""
    import torch
    q, k, v = qkv(80, 1, 4, 2, 300, 64, "fp16")
    dout = torch.zeros_like(q)
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    out = [torch.empty_like(x) for x in (q, k, v)]
    ws = torch.empty(bd.attn_window_bwd_workspace_size(1, 4, 2, 300, 64, 90, 3), dtype=torch.uint8, device="cuda")

    def step():
        bd.sage_attn_window_fwd(q, k, v, window=90, sinks=3, out=o, lse_out=lse)
        bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=90, sinks=3, workspace=ws, out=out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    g = gen(81)
    for i in range(4):
        for x in (q, k, v, dout):
            x.copy_(randn(g, *x.shape))
        graph.replay()
        oe, le = bd.sage_attn_window_fwd(q, k, v, window=90, sinks=3)
        ge = bd.sage_attn_window_bwd(q, k, v, oe, le, dout, window=90, sinks=3)
        torch.cuda.synchronize()
        assert torch.equal(o, oe) and torch.equal(lse, le) and all(torch.equal(a, b) for a, b in zip(out, ge)), i


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_window_forward_strides(dtype):
    """[B, N, H, D] tensors, heads broadcast from one, a slice of a longer buffer, an output of other
    strides and without L: the same bits as for contiguous copies."""
    import torch
    B, H, N, D = 2, 4, 150, 64
    q, k, v = qkv(5, B, H, H, N, D, dtype)
    ref, lref = bd.sage_attn_window_fwd(q, k, v, window=40, sinks=3)
    tr = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v)]
    out = torch.full((B, N, H, D), 7.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    o, lse = bd.sage_attn_window_fwd(*tr, window=40, sinks=3, out=out)
    assert o is out and torch.equal(o, ref) and torch.equal(lse, lref)
    o, lse = bd.sage_attn_window_fwd(*tr, window=40, sinks=3, lse=False)
    assert lse is None and torch.equal(o, ref)
    big = torch.randn((B, H, 2 * N + 9, D + 16), device="cuda").to(q.dtype)
    sl = big[:, :, 4:4 + N, 8:8 + D]
    sl.copy_(k)
    assert torch.equal(bd.sage_attn_window_fwd(q, sl, v, window=40, sinks=3)[0], ref)
    one = k[:, :1].expand(B, H, N, D)
    want = bd.sage_attn_window_fwd(q, one.contiguous(), v[:, :1].expand(B, H, N, D).contiguous(), window=40)
    got = bd.sage_attn_window_fwd(q, one, v[:, :1].expand(B, H, N, D), window=40)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # the same head grouped instead of broadcast
    assert torch.equal(bd.sage_attn_window_fwd(q, k[:, :1], v[:, :1], window=40)[0], want[0])
    # every token the same key (token stride 0)
    rep = k[:, :, :1].expand(B, H, N, D)
    assert torch.equal(bd.sage_attn_window_fwd(q, rep, v, window=40)[0], bd.sage_attn_window_fwd(q, rep.contiguous(), v, window=40)[0])


@pytest.mark.parametrize("D", [64, 128])
def test_window_forward_large_scores(D):
    """Scores of hundreds, of which one key takes all; and rows whose scores are all very low."""
    import torch
    q, k, v = qkv(9, 1, 2, 2, 200, D, "bf16")
    for scale in (30.0, -30.0):
        qs = (q * scale)
        o, lse = bd.sage_attn_window_fwd(qs, k, v, window=64, sinks=2)
        check_window(qs, k, v, o, lse, 64, 2, None, "scores x %g" % scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_window_forward_ignores_what_it_does_not_see(D, dtype):
    """NaN and infinity in K, V and Q behind a sequence's end, and in K and V of tokens that a row
    does not see (future ones, ones before its window): its bits stay.  Rows that see them get them."""
    import torch
    B, Hq, Hkv, N = 2, 4, 2, 300
    q, k, v = qkv(40 + D, B, Hq, Hkv, N, D, dtype)
    lens = torch.tensor([300, 170], dtype=torch.int32, device="cuda")
    for window, sinks in ((None, 0), (70, 4)):
        ref = bd.sage_attn_window_fwd(q, k, v, window=window, sinks=sinks, lens=lens)
        for bad in (float("nan"), float("inf"), -float("inf")):
            qb, kb, vb = q.clone(), k.clone(), v.clone()
            for x in (qb, kb, vb):
                x[1, :, 170:] = bad
            got = bd.sage_attn_window_fwd(qb, kb, vb, window=window, sinks=sinks, lens=lens)
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
            for at in (10, 200):
                for what in ("k", "v"):
                    kb, vb = k.clone(), v.clone()
                    (kb if what == "k" else vb)[0, 1, at, D // 2 if what == "v" else slice(None)] = bad
                    o, lse = bd.sage_attn_window_fwd(q, kb, vb, window=window, sinks=sinks, lens=lens)
                    torch.cuda.synchronize()
                    i = torch.arange(N, device="cuda")
                    sees = _lm.visible(i, at, 300, window, sinks)
                    assert torch.equal(o[1], ref[0][1]) and torch.equal(o[0, :2], ref[0][0, :2])
                    assert torch.equal(o[0, 2:, ~sees], ref[0][0, 2:, ~sees]) and torch.equal(lse[0, 2:, ~sees], ref[1][0, 2:, ~sees])
                    if what == "v":
                        c = o[0, 2:, :, D // 2]
                        assert torch.equal(c[:, sees].float().nan_to_num(7, 8, 9), torch.full_like(c[:, sees].float(), bad).nan_to_num(7, 8, 9))
                        c = torch.arange(D, device="cuda") != D // 2
                        assert torch.equal(o[..., c], ref[0][..., c]) and torch.equal(lse, ref[1])


# ---------------------------------------------------------------- the cache
def make_cache(g, S, Hkv, page, D, lens, dtype, int8, layout="hnd", spare=3, fill=None):
    """A cache with random pages for sequences of these lengths; returns its tensors and the table."""
    import torch
    dt = getattr(torch, DT[dtype])
    M = max(1, max(-(-max(0, n) // page) for n in lens))
    P = S * M + spare
    shape = (P, Hkv, page, D)
    k, v = randn(g, *shape) + randn(g, 1, Hkv, 1, D), randn(g, *shape)
    ks = vs = None
    if int8:
        (k, ks), (v, vs) = _lm.quantized(k.to(dt)), _lm.quantized(v.to(dt))
    else:
        k, v = k.to(dt), v.to(dt)
    if layout == "nhd":
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    table = perm[:S * M].view(S, M).contiguous()
    return dict(k_cache=k, v_cache=v, k_scale=ks, v_scale=vs), table, perm[S * M:]


def check_decode(q, c, table, lens, window, sinks, o, lse, w0, w1, label):
    import torch
    S, Hq, D = q.shape
    Hkv, page = c["k_cache"].shape[1:3]
    G, u = Hq // Hkv, _lm.unit(q.dtype)
    up = (_lm.unit(torch.bfloat16) if c["k_scale"] is not None else u) ** 2   # P in two parts
    tab = table.cpu()
    worst = [0.0, 0.0, 0.0]
    for s in range(S):
        n = max(0, min(int(lens[s]), table.shape[1] * page))
        for h in range(Hkv):
            kr, has = _lm.cache_rows(c["k_cache"], c["k_scale"], tab[s], h, n)
            vr, _ = _lm.cache_rows(c["v_cache"], c["v_scale"], tab[s], h, n)
            hs = slice(h * G, (h + 1) * G)
            r = _lm.decode_attention(q[s, hs].double(), kr, vr, has.to(q.device), window, sinks)
            r["e"] = r["e"] * 1.1 + 2.0 ** -22 * r["e"].clamp(min=0) / 2.0 ** -24 / (D + 4)   # the scale's product
            t = _lm.o_bound(r, n, u, up)
            worst[0] = max(worst[0], float(((o[s, hs].double() - r["o"]).abs() / t).max()))
            if lse is not None:
                d = lse[s, hs].double() - r["lse"]
                dead = r["lse"] == -math.inf
                assert bool((lse[s, hs][dead] == -math.inf).all()), label
                d = torch.where(dead, 0.0, d).abs()
                worst[1] = max(worst[1], float((d / _lm.lse_bound(r, n)).max()))
            if w1 is not None and n:
                want = w0[s, h, :n].double() + r["p"].sum(0)
                rel = (2 * r["e"] + (n + 64) * 2.0 ** -23)
                tol = (rel * r["p"]).sum(0) + (G + 2) * 2.0 ** -24 * want.abs() + 1e-30
                worst[2] = max(worst[2], float(((w1[s, h, :n].double() - want).abs() / tol).max()))
        if w1 is not None:
            assert torch.equal(w1[s, :, n:], w0[s, :, n:]), label
    say("%s: O at %.3f of its bound, L at %.3f, weights at %.3f" % (label, *worst))
    assert max(worst) <= 1, label


DECODES = [
    # Hq, Hkv, page, D, lens, dtype, int8, layout, window, sinks, weights
    (1, 1, 16, 64, [1], "bf16", False, "hnd", None, 0, False),
    (8, 2, 16, 64, [77], "fp16", False, "hnd", None, 0, True),
    (8, 8, 1, 128, [40, 3], "bf16", False, "hnd", None, 0, False),
    (4, 1, 24, 128, [100, 0, 25], "bf16", False, "nhd", None, 0, True),
    (32, 8, 64, 128, [700, 1, 512, 513], "bf16", False, "hnd", None, 0, True),
    (20, 1, 32, 128, [300, 900], "fp16", False, "nhd", None, 0, True),
    (64, 2, 128, 64, [1000, 130], "bf16", True, "hnd", None, 0, True),
    (16, 1, 16, 128, [650, 31, 32, 33, 640], "fp16", True, "hnd", None, 0, False),
    (6, 2, 256, 128, [2000], "bf16", True, "nhd", 128, 4, True),
    (8, 2, 32, 128, [1500, 64, 9], "bf16", False, "hnd", 100, 4, True),
    (8, 8, 48, 64, [1200, 600], "fp16", False, "hnd", 1, 0, False),
    (4, 4, 64, 128, [1300, 0, 0, 640], "bf16", False, "hnd", 257, 70, True),
    (4, 2, 16, 64, [900, 8], "fp16", True, "hnd", 64, 1, True),
]


@pytest.mark.parametrize("case", DECODES)
def test_paged_decode(case):
    import torch
    Hq, Hkv, page, D, lens, dtype, int8, layout, window, sinks, weights = case
    g = gen(100 + sum(lens) + D)
    S = len(lens)
    c, table, _ = make_cache(g, S, Hkv, page, D, lens, dtype, int8, layout)
    q = randn(g, S, Hq, D).to(getattr(torch, DT[dtype]))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    w0 = torch.rand((S, Hkv, table.shape[1] * page + 5), generator=g, device="cuda")
    w1 = w0.clone() if weights else None
    say("decode %s" % (case,))
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, window=window, sinks=sinks,
                                       k_scale=c["k_scale"], v_scale=c["v_scale"], weights=w1)
    torch.cuda.synchronize()
    check_decode(q, c, table, lens, window, sinks, o, lse, w0, w1, "decode %s" % (case,))
    w2 = w0.clone() if weights else None
    o2, lse2 = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, window=window, sinks=sinks,
                                         k_scale=c["k_scale"], v_scale=c["v_scale"], weights=w2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and (w1 is None or torch.equal(w1, w2))


@pytest.mark.parametrize("S,Hkv,empty", [(64, 4, False), (65, 1, False), (150, 2, True), (5000, 1, True)])
def test_paged_decode_many_ragged_sequences(S, Hkv, empty):
    """More sequences than a wave counts at a time, runs of empty ones among them: every one as if it
    were alone (up to the rounding of the split)."""
    import torch
    g = gen(3)
    page, D = 16, 64
    lens = [int(x) for x in np.random.default_rng(4).integers(0, 900, S)]
    lens[0], lens[62], lens[-1] = 0, 899, 0
    if empty:
        lens[64:130] = [0] * 66
        lens[1:3] = [0, 0]
    c, table, _ = make_cache(g, S, Hkv, page, D, lens, "bf16", False)
    q = randn(g, S, 4, D).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln)
    torch.cuda.synchronize()
    pick = sorted({i % S for i in (0, 1, 2, 3, 31, 62, 63, 64, 65, 127, 128, 129, 130, 131, S // 2, -3, -2, -1)})
    sub = torch.tensor(pick, device="cuda")
    check_decode(q[sub], c, table[sub], [lens[i] for i in pick], None, 0, o[sub], lse[sub], None, None, "%d sequences" % S)


@pytest.mark.parametrize("int8", [False, True])
def test_paged_decode_ignores_what_it_does_not_see(int8):
    """NaN and infinity in unused slots, pages and scales, table entries behind a sequence's end that
    are no pages: the same bits.  Entries that are no pages inside it: their tokens are not seen."""
    import torch
    g = gen(8)
    lens, page = [70, 33, 600], 32
    c, table, spare = make_cache(g, 3, 2, page, 128, lens, "bf16", int8)
    q = randn(g, 3, 8, 128).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = dict(window=200, sinks=3, k_scale=c["k_scale"], v_scale=c["v_scale"])
    ref = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, **args)
    used = torch.zeros(c["k_cache"].shape[0], page, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for j in range(n):
            if _lm.visible(n - 1, torch.tensor(j), n, 200, 3):
                used[int(table[s, j // page]), j % page] = True
    for bad in (float("nan"), float("inf"), -float("inf")):
        for x in ("k_scale", "v_scale") if int8 else ("k_cache", "v_cache"):
            m = ~used[:, None, :] if int8 else ~used[:, None, :, None]
            c[x].masked_fill_(m, bad)
        for t in (-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1):
            tb = table.clone()
            for s, n in enumerate(lens):
                tb[s, -(-n // page):] = t
            got = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], tb, ln, **args)
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
    tb = table.clone()
    tb[2, 18], tb[2, 0], tb[0, :] = -1, c["k_cache"].shape[0], 2 ** 31 - 1
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], tb, ln, **args)
    torch.cuda.synchronize()
    assert torch.equal(o[1], ref[0][1]) and bool((o[0] == 0).all()) and bool((lse[0] == -math.inf).all())
    c = {k: (x.nan_to_num(0, 0, 0) if x is not None and x.is_floating_point() else x) for k, x in c.items()}
    check_decode(q, c, tb, lens, 200, 3, o, lse, None, None, "bad pages")


def test_paged_decode_shared_pages_strides_and_lengths():
    """Sequences that share their first pages; q of other strides; lengths beyond the table's
    capacity or negative."""
    import torch
    g = gen(12)
    c, table, _ = make_cache(g, 3, 2, 16, 64, [160, 160, 160], "fp16", False)
    table[1, :5] = table[0, :5]
    table[2] = table[0]
    q = randn(g, 3, 4, 64).half()
    lens = [155, 90, 155]
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    big = torch.zeros((3, 4, 2, 64), dtype=torch.float16, device="cuda")
    big[:, :, 1] = q
    w0 = torch.zeros((3, 2, 160), device="cuda")
    w = w0.clone()
    o, lse = bd.sage_attn_paged_decode(big[:, :, 1], c["k_cache"], c["v_cache"], table, ln, weights=w)
    torch.cuda.synchronize()
    check_decode(q, c, table, lens, None, 0, o, lse, w0, w, "shared pages")
    o2, _ = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, torch.tensor([10 ** 9, -3, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    o3, _ = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, torch.tensor([160, 0, 160], dtype=torch.int32, device="cuda"))
    assert torch.equal(o2, o3) and bool((o2[1] == 0).all())


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,D,page,N", [("bf16", 128, 16, 1), ("fp16", 64, 24, 50), ("bf16", 64, 1, 7), ("fp16", 128, 64, 131)])
def test_append(dtype, D, page, N, layout, int8):
    """The stored rows, bit for bit; every other slot as it was."""
    import torch
    g = gen(N + D)
    S, Hkv = 4, 3
    dt = getattr(torch, DT[dtype])
    c, table, _ = make_cache(g, S, Hkv, page, D, [N + 40] * S, dtype, int8, layout)
    cap = table.shape[1] * page
    pos = torch.tensor([0, 13, cap - 2, 40], dtype=torch.int32, device="cuda")
    counts = torch.tensor([N, max(0, N - 3), N, -1], dtype=torch.int32, device="cuda")
    table[1, 14 // page] = -1                            # no page for these: not stored
    k = randn(g, S, N, Hkv, D).to(dt).transpose(1, 2)
    v = randn(g, S, Hkv, N, D).to(dt)
    k[0, 0, 0] = 0
    v[0, 1, 0] *= 1e-4
    w = torch.ones((S, Hkv, cap + 3), device="cuda")
    want = {x: t.clone() if t is not None else None for x, t in c.items()}
    ww = w.clone()
    for s in range(S):
        for t in range(min(N, max(0, int(counts[s])))):
            j = int(pos[s]) + t
            pid = int(table[s, j // page]) if j < cap else -1
            if not 0 <= pid < c["k_cache"].shape[0]:
                continue
            ww[s, :, j] = 0
            for x, cc, sc in ((k, "k_cache", "k_scale"), (v, "v_cache", "v_scale")):
                row = x[s, :, t]
                if int8:
                    row, want[sc][pid, :, j % page] = _lm.quantized(row)
                want[cc][pid, :, j % page] = row
    bd.sage_kv_append(k, v, c["k_cache"], c["v_cache"], table, pos, counts, k_scale=c["k_scale"], v_scale=c["v_scale"], weights=w)
    torch.cuda.synchronize()
    for x in c:
        assert c[x] is None or torch.equal(c[x], want[x]), x
    assert torch.equal(w, ww)


def test_append_tiny_and_large_rows_in_8_bits():
    """Rows of subnormals have scale 0; the largest fp16 and bf16 values keep their codes."""
    import torch
    for dt, big in ((torch.float16, 65504.0), (torch.bfloat16, 3e38)):
        x = torch.zeros((1, 1, 4, 64), dtype=dt, device="cuda")
        x[0, 0, 0] = torch.finfo(dt).smallest_normal / 64 if dt == torch.bfloat16 else 6e-8
        x[0, 0, 1, 3], x[0, 0, 1, 4] = big, -big
        x[0, 0, 2, 0] = 1.0
        kc = torch.zeros((1, 1, 4, 64), dtype=torch.int8, device="cuda")
        ks = torch.zeros((1, 1, 4), device="cuda")
        vc, vs = kc.clone(), ks.clone()
        z = torch.zeros((1,), dtype=torch.int32, device="cuda")
        bd.sage_kv_append(x, x, kc, vc, z.view(1, 1), z, k_scale=ks, v_scale=vs)
        codes, s = _lm.quantized(x)
        assert torch.equal(kc, codes) and torch.equal(ks, s) and torch.equal(vc, codes) and torch.equal(vs, s)


EVICTS = [
    # Hkv, page, D, lens, budget, first, last, dtype, int8
    (1, 16, 64, [1], 1, 0, 0, "bf16", False),
    (2, 16, 64, [100, 40, 0, 41], 40, 4, 8, "fp16", False),
    (2, 24, 128, [5000, 999, 1000, 1001], 1000, 16, 300, "bf16", False),
    (3, 32, 128, [3000, 2049], 2048, 0, 2048, "bf16", True),
    (1, 1, 64, [77, 30], 20, 20, 0, "bf16", True),
    (2, 64, 128, [700], 699, 0, 0, "fp16", False),
    (1, 128, 128, [40000], 1, 0, 0, "bf16", False),
    (2, 64, 64, [40001, 9000, 16385], 9001, 8200, 100, "bf16", False),
    (1, 256, 64, [200000], 150000, 3, 20000, "fp16", True),
    (1, 32, 64, [20000], 300, 100, 200, "fp16", False),
]


@pytest.mark.parametrize("kind", ["normal", "ties", "odd"])
@pytest.mark.parametrize("case", EVICTS)
def test_evict(case, kind):
    import torch
    Hkv, page, D, lens, budget, first, last, dtype, int8 = case
    g = gen(sum(lens) + budget)
    S = len(lens)
    c, table, _ = make_cache(g, S, Hkv, page, D, lens, dtype, int8, "nhd" if page == 24 else "hnd")
    M2 = -(-budget // page)
    for x in c:                                          # pages for the kept tokens
        if c[x] is not None:
            more = torch.zeros((S * M2,) + tuple(c[x].shape[1:]), dtype=c[x].dtype, device="cuda")
            c[x] = torch.cat([c[x], more])
    P = c["k_cache"].shape[0]
    new_table = torch.arange(P - S * M2, P, dtype=torch.int32, device="cuda").flip(0).view(S, M2).contiguous()
    cap = table.shape[1] * page
    w = torch.exp(3 * randn(g, S, Hkv, cap + 7) - 6)
    if kind == "ties":
        w = torch.round(w * 4) / 4
    if kind == "odd":
        w = randn(g, S, Hkv, cap + 7)
        r = torch.rand(w.shape, generator=g, device="cuda")
        for lo, x in ((0.0, float("nan")), (0.02, float("inf")), (0.04, -float("inf")), (0.06, 0.0), (0.2, -0.0), (0.35, 1e-42)):
            w = torch.where((r >= lo) & (r < lo + 0.02 if lo < 0.06 else r >= lo), x, w) if lo < 0.06 else torch.where(
                (r >= lo) & (r < lo + 0.1), x, w)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = {x: t.clone() if t is not None else None for x, t in c.items()}
    say("evict %s %s" % (case, kind))
    nl, nw, kept = bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, w, new_table, budget, first, last,
                                    k_scale=c["k_scale"], v_scale=c["v_scale"])
    torch.cuda.synchronize()
    assert nl.tolist() == [min(n, budget) for n in lens]
    wc, tc, ntc = w.cpu().numpy(), table.cpu().numpy(), new_table.cpu().numpy()
    for s, n in enumerate(lens):
        for h in range(Hkv):
            keep = _lm.kept_tokens(wc[s, h, :n], n, budget, first, last)
            m = len(keep)
            got = kept[s, h].cpu().numpy()
            assert np.array_equal(got[:m], keep) and (got[m:] == -1).all(), (s, h)
            nwc = nw[s, h].cpu().numpy()
            assert np.array_equal(nwc[:m].view(np.int32), wc[s, h, keep].view(np.int32)) and (nwc[m:] == 0).all()
            sp, so = (torch.from_numpy(np.ascontiguousarray(x)).long().cuda() for x in (tc[s, keep // page], keep % page))
            j = np.arange(m)
            dp, do = (torch.from_numpy(np.ascontiguousarray(x)).long().cuda() for x in (ntc[s, j // page], j % page))
            for x in want:
                if want[x] is not None:
                    want[x][dp, h, do] = want[x][sp, h, so]
    for x in c:
        assert c[x] is None or torch.equal(c[x], want[x]), x


def test_evict_in_place_for_short_sequences_and_bad_pages():
    """A sequence within its budget may keep its pages; tokens without a page are not moved."""
    import torch
    g = gen(2)
    c, table, spare = make_cache(g, 2, 2, 16, 64, [30, 64], "bf16", False, spare=4)
    new_table = table[:, :2].contiguous()
    new_table[1] = spare[:2]
    table[1, 1] = -5
    before = {x: t.clone() for x, t in c.items() if t is not None}
    w = torch.rand((2, 2, 64), generator=g, device="cuda")
    ln = torch.tensor([30, 64], dtype=torch.int32, device="cuda")
    nl, nw, kept = bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, w, new_table, 32, 16, 16)
    torch.cuda.synchronize()
    assert nl.tolist() == [30, 32]
    assert torch.equal(kept[1, 0].cpu(), torch.cat([torch.arange(16), torch.arange(48, 64)]).int())
    for x in before:
        a, b = c[x], before[x]
        assert torch.equal(a[table[0].long()], b[table[0].long()])
        assert torch.equal(a[spare[0].long()], b[table[1, 0].long()]) and torch.equal(a[spare[1].long()], b[table[1, 3].long()])
    new_table[1, 0] = c["k_cache"].shape[0]
    again = {x: t.clone() for x, t in c.items() if t is not None}
    bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, w, new_table, 32, 16, 16)
    torch.cuda.synchronize()
    assert all(torch.equal(c[x], again[x]) for x in again)


@pytest.mark.parametrize("int8", [False, True])
def test_caches_beyond_32_bit_offsets(int8):
    """Pages behind 2^32 elements of the cache: stored, read and moved as in a small one."""
    import torch
    g = gen(51)
    S, Hkv, page, D, lens = 2, 16, 256, 128, [700, 513]
    c, table, spare = make_cache(g, S, Hkv, page, D, lens, "bf16", int8)
    q = randn(g, S, 32, D).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kn, vn = (randn(g, S, Hkv, 1, D).to(torch.bfloat16) for _ in range(2))
    w = torch.rand((S, Hkv, table.shape[1] * page), generator=g, device="cuda")
    new_table = spare[:2].view(2, 1).contiguous()
    P, n = c["k_cache"].shape[0], 2 ** 32 // (Hkv * page * D)
    big = {}
    for x, t in c.items():
        big[x] = None
        if t is not None:                                # the same pages, n places further on
            big[x] = torch.empty((n + P,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda")
            big[x][n:] = t
    outs = []
    for cc, off in ((c, 0), (big, n)):
        tb, nt, ww = table + off, new_table + off, w.clone()
        kw = dict(k_scale=cc["k_scale"], v_scale=cc["v_scale"])
        args = (cc["k_cache"], cc["v_cache"], tb)
        bd.sage_kv_append(kn, vn, *args, ln - 1, weights=ww, **kw)
        o, lse = bd.sage_attn_paged_decode(q, *args, ln, weights=ww, **kw)
        ev = bd.sage_kv_evict(*args, ln, ww, nt, 200, 3, 50, **kw)
        o2, lse2 = bd.sage_attn_paged_decode(q, cc["k_cache"], cc["v_cache"], nt, ev[0], **kw)
        torch.cuda.synchronize()
        outs.append((o, lse, ww, *ev, o2, lse2))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for x in c:
        assert c[x] is None or torch.equal(big[x][n:], c[x])
    del big


def test_binding_refuses_mismatched_tensors():
    import torch
    q, k, v = qkv(1, 2, 4, 2, 64, 64, "bf16")
    g = gen(1)
    c, table, _ = make_cache(g, 2, 2, 16, 64, [40, 20], "bf16", False)
    c8, _, _ = make_cache(g, 2, 2, 16, 64, [40, 20], "bf16", True)
    kc, vc = c["k_cache"], c["v_cache"]
    ln = torch.tensor([40, 20], dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_window_fwd(q, k, v)
    w = torch.zeros((2, 2, 48), device="cuda")
    bad = [
        lambda: bd.sage_attn_window_fwd(q, k.half(), v),
        lambda: bd.sage_attn_window_fwd(q, k[:, :, :-1], v),
        lambda: bd.sage_attn_window_fwd(q, torch.cat([k, k[:, :1]], 1), torch.cat([v, v[:, :1]], 1)),
        lambda: bd.sage_attn_window_fwd(q[..., 1:], k[..., 1:], v[..., 1:]),
        lambda: bd.sage_attn_window_fwd(q, k, v, window=0),
        lambda: bd.sage_attn_window_fwd(q, k, v, sinks=-1),
        lambda: bd.sage_attn_window_fwd(q, k, v, lens=ln.long()),
        lambda: bd.sage_attn_window_fwd(q, k, v, lens=ln[:1]),
        lambda: bd.sage_attn_window_fwd(q, k, v, out=torch.empty_like(q).float()),
        lambda: bd.sage_attn_window_fwd(q, k, v, lse_out=lse[:, :1]),
        lambda: bd.sage_attn_window_bwd(q, k, v, o, lse.half(), q),
        lambda: bd.sage_attn_window_bwd(q, k, v, o.float(), lse, q),
        lambda: bd.sage_attn_window_bwd(q, k, v, o, lse, k),
        lambda: bd.sage_attn_window_bwd(q, k, v, o, lse, q, out=(q, k, v.float())),
        lambda: bd.sage_attn_window_bwd(q, k, v, o, lse, q, workspace=torch.empty(9, device="cuda")),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0].half(), kc, vc, table, ln),
        lambda: bd.sage_attn_paged_decode(q[:, :3, 0], kc, vc, table, ln),
        lambda: bd.sage_attn_paged_decode(q[:1, :, 0], kc, vc, table, ln),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc[:-1], table, ln),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table.long(), ln),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table.t(), ln),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table, ln.cpu()),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table, ln, weights=w[:, :, :47]),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table, ln, weights=w.double()),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], c8["k_cache"], c8["v_cache"], table, ln),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], kc, vc, table, ln, k_scale=c8["k_scale"], v_scale=c8["v_scale"]),
        lambda: bd.sage_attn_paged_decode(q[:, :, 0], c8["k_cache"], c8["v_cache"], table, ln, k_scale=c8["k_scale"], v_scale=c8["v_scale"].half()),
        lambda: bd.sage_kv_append(k.half(), v.half(), kc, vc, table, ln),
        lambda: bd.sage_kv_append(k, v[:, :, 1:], kc, vc, table, ln),
        lambda: bd.sage_kv_append(k[:1], v[:1], kc, vc, table, ln),
        lambda: bd.sage_kv_append(k, v, kc, vc, table, ln[:1]),
        lambda: bd.sage_kv_append(k, v, kc, vc, table, ln, counts=ln.float()),
        lambda: bd.sage_kv_evict(kc, vc, table, ln, w, table[:, :1].contiguous(), 17),
        lambda: bd.sage_kv_evict(kc, vc, table, ln, w, table[:1], 16),
        lambda: bd.sage_kv_evict(kc, vc, table, ln, w[:, :1], table, 16),
        lambda: bd.sage_kv_evict(kc, vc, table, ln, w, table, 16, 9, 8),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            f()
            raise AssertionError(i)
    # the library's own refusals come through as SageError
    with pytest.raises(bd.SageError):
        bd.sage_kv_append(k, v, kc[:1].expand(kc.shape), vc, table, ln)      # pages that are one and the same
    with pytest.raises(bd.SageError):
        bd.sage_attn_window_fwd(q, k, v, out=q[:, :1].expand(q.shape))
    with pytest.raises(bd.SageError):
        bd.sage_attn_window_bwd(q, k, v, o, lse, q, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("int8", [False, True])
def test_prompt_tokens_and_eviction_together(int8):
    """A padded batch of prompts through the window attention, its keys stored, then tokens one at a
    time through the cache: each row is the window attention's over the whole sequence.  Then an
    eviction by the weights added up on the way, and a token over what is left."""
    import torch
    g = gen(77)
    S, Hq, Hkv, N, T, D, page = 3, 8, 2, 90, 12, 64, 16
    lens0 = [90, 41, 7]
    q, k, v = qkv(21, S, Hq, Hkv, N + T, D, "bf16")
    window, sinks = 64, 4
    if int8:                                             # what the cache will hold stands for these
        (kc, ks), (vc, vs) = _lm.quantized(k), _lm.quantized(v)
    M = -(-(N + T) // page)
    c, table, spare = make_cache(g, S, Hkv, page, D, [M * page] * S, "bf16", int8, spare=3 * S)
    kw = dict(k_scale=c["k_scale"], v_scale=c["v_scale"])
    pos = torch.zeros(S, dtype=torch.int32, device="cuda")
    counts = torch.tensor(lens0, dtype=torch.int32, device="cuda")
    w = torch.full((S, Hkv, M * page), 9.0, device="cuda")
    o, _ = bd.sage_attn_window_fwd(q[:, :, :N], k[:, :, :N], v[:, :, :N], window=window, sinks=sinks, lens=counts)
    bd.sage_kv_append(k[:, :, :N], v[:, :, :N], c["k_cache"], c["v_cache"], table, pos, counts, weights=w, **kw)
    check_window(q[:, :, :N], k[:, :, :N], v[:, :, :N], o, None, window, sinks, lens0, "prompts")
    lens = counts.clone()
    for t in range(T):                                   # every sequence goes on with its own next token
        at = lens.long()
        b = torch.arange(S, device="cuda")
        qt, kt, vt = q[b, :, at], k[b, :, at], v[b, :, at]
        bd.sage_kv_append(kt[:, :, None], vt[:, :, None], c["k_cache"], c["v_cache"], table, lens, weights=w, **kw)
        lens = lens + 1
        w0 = w.clone()
        o, lse = bd.sage_attn_paged_decode(qt, c["k_cache"], c["v_cache"], table, lens, window=window, sinks=sinks, weights=w, **kw)
        torch.cuda.synchronize()
        check_decode(qt, c, table, lens.tolist(), window, sinks, o, lse, w0, w, "token %d" % t)
        full = (kc * ks[..., None], vc * vs[..., None]) if int8 else (k.double(), v.double())
        for s in range(S):
            n = int(lens[s])
            r = _lm.window_attention(q[s, 3].double()[:n], full[0][s, 0].double()[:n], full[1][s, 0].double()[:n], window, sinks, n)
            assert float((o[s, 3].double() - r["o"][-1]).abs().max()) <= 2.0 ** -6 * float(r["av"][-1].max())
    for s in range(S):
        assert bool((w[s, :, int(lens[s]):] == 9).all()) and bool((w[s, :, :lens0[s]] >= 0).all())
    # each step's weights sum to the group's heads
    tot = torch.stack([w[s, :, :int(lens[s])].sum(-1) for s in range(S)])
    assert float((tot - T * Hq // Hkv).abs().max()) < 1e-3 * T * Hq
    budget = 40
    new_table = spare[:3 * S].view(S, 3).contiguous()
    nl, nw, kept = bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, lens, w, new_table, budget, 4, 16, **kw)
    qn = randn(g, S, Hq, D).to(torch.bfloat16)
    o, lse = bd.sage_attn_paged_decode(qn, c["k_cache"], c["v_cache"], new_table, nl, **kw)
    torch.cuda.synchronize()
    check_decode(qn, c, new_table, nl.tolist(), None, 0, o, lse, None, None, "after the eviction")
    for s in range(S):
        m = int(nl[s])
        for h in range(Hkv):
            a, _ = _lm.cache_rows(c["k_cache"], c["k_scale"], new_table[s].cpu(), h, m)
            b, _ = _lm.cache_rows(c["k_cache"], c["k_scale"], table[s].cpu(), h, int(lens[s]))
            assert torch.equal(a, b[kept[s, h, :m].long()])
            assert torch.equal(nw[s, h, :m], w[s, h][kept[s, h, :m].long()])


def test_calls_on_two_streams_at_once():
    """Training and decoding of different inputs interleaved on two streams: each as alone."""
    import torch
    jobs = []
    for i in range(2):
        q, k, v = qkv(300 + i, 2, 8, 2, 400, 64, "bf16")
        dout = randn(gen(310 + i), *q.shape).to(q.dtype)
        g = gen(320 + i)
        c, table, _ = make_cache(g, 3, 2, 16, 128, [900, 700, 800], "bf16", bool(i))
        qd = randn(g, 3, 8, 128).to(torch.bfloat16)
        ln = torch.tensor([900, 700 - 300 * i, 800], dtype=torch.int32, device="cuda")

        def job(q=q, k=k, v=v, dout=dout, c=c, table=table, qd=qd, ln=ln):
            o, lse = bd.sage_attn_window_fwd(q, k, v, window=90, sinks=4)
            grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=90, sinks=4)
            w = torch.zeros((3, 2, table.shape[1] * 16), device="cuda")
            d = bd.sage_attn_paged_decode(qd, c["k_cache"], c["v_cache"], table, ln, k_scale=c["k_scale"], v_scale=c["v_scale"], weights=w)
            return (o, lse, *grads, *d, w)

        jobs.append((job, job(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (job, _, s) in enumerate(jobs):
            with torch.cuda.stream(s):
                got[i].append(job())
    torch.cuda.synchronize()
    for i, (_, ref, _) in enumerate(jobs):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, ref)), i


def test_captured_steps_follow_the_lengths_and_streams():
    """Append and decode captured into a graph on another stream; replayed several times with lengths
    that grow on the device, eager work between the replays: each as the eager calls."""
    import torch
    g = gen(31)
    S, Hq, Hkv, D, page = 5, 8, 2, 128, 16
    start = [0, 700, 15, 333, 40]
    c, table, _ = make_cache(g, S, Hkv, page, D, [720] * S, "bf16", False)
    eager = {x: t.clone() if t is not None else None for x, t in c.items()}
    cap = table.shape[1] * page
    lens = torch.tensor(start, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((S, h, 1, D), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    w = torch.zeros((S, Hkv, cap), device="cuda")
    we = w.clone()
    o = torch.empty((S, Hq, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((S, Hq), device="cuda")
    ws = torch.empty(bd.attn_paged_decode_workspace_size(S, Hq, Hkv, D, table.shape[1], page, True), dtype=torch.uint8, device="cuda")

    def step():
        bd.sage_kv_append(k, v, c["k_cache"], c["v_cache"], table, lens, weights=w)
        lens.add_(1)
        bd.sage_attn_paged_decode(q[:, :, 0], c["k_cache"], c["v_cache"], table, lens, weights=w, out=o, lse_out=lse, workspace=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    torch.cuda.synchronize()
    lens.copy_(torch.tensor(start, dtype=torch.int32))
    w.zero_()
    le = lens.clone()
    for x in ("k_cache", "v_cache"):
        c[x].copy_(eager[x])
    for i in range(6):
        for t in (q, k, v):
            t.copy_(randn(g, *t.shape))
        graph.replay()
        bd.sage_kv_append(k, v, eager["k_cache"], eager["v_cache"], table, le, weights=we)
        le = le + 1
        oe, lsee = bd.sage_attn_paged_decode(q[:, :, 0], eager["k_cache"], eager["v_cache"], table, le, weights=we)
        torch.cuda.synchronize()
        assert torch.equal(o, oe) and torch.equal(lse, lsee) and torch.equal(w, we) and torch.equal(lens, le), i
        assert all(torch.equal(c[x], eager[x]) for x in ("k_cache", "v_cache")), i
