"""GPU checks of the norms with rotation, the MXFP4 cache with the attention over it, and page tables
against their definitions in 64 bits (_more_lm.py, which derives the bounds)."""
import math

import numpy as np
import pytest

from paper_2505_11594_amd import binding as bd

import _lm
import _more_lm as mo
from _gpu import torch_dev, say

pytestmark = pytest.mark.gpu

DT = {"bf16": "bfloat16", "fp16": "float16"}


def gen(seed):
    torch = torch_dev()
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda")


# ---------------------------------------------------------------- norms with rotation
ROPES = [
    # B, Hq, Hkv, N, D, R, pairs, dtype, pos, lens, packed, weights
    (1, 1, 1, 1, 64, 64, False, "bf16", "0", None, False, True),
    (1, 1, 1, 1, 128, 128, True, "fp16", "each", None, False, True),
    (3, 32, 8, 1, 128, 128, False, "bf16", "start", None, True, True),
    (2, 6, 2, 37, 128, 128, False, "fp16", "0", [37, 5], True, True),
    (4, 24, 24, 101, 64, 32, True, "fp16", "start", [101, 0, 64, 1], True, True),
    (2, 7, 1, 50, 64, 24, False, "bf16", "each", [50, 33], False, True),
    (1, 14, 2, 200, 128, 8, False, "bf16", "far", None, True, False),
    (1, 20, 4, 65, 128, 96, True, "bf16", "far", None, True, True),
    (2, 64, 16, 129, 64, 64, False, "fp16", "each", None, False, False),
    (1, 3, 3, 300, 128, 0, False, "bf16", "0", [299], False, True),
    (1, 16, 1, 5000, 64, 64, False, "bf16", "0", None, True, True),
]


def rope_case(case):
    import torch
    B, Hq, Hkv, N, D, R, pairs, dtype, at, lens, packed, weights = case
    g = gen(7 + N + 3 * D + R)
    dt = getattr(torch, DT[dtype])
    if packed:                                           # views of one projection
        x = randn(g, B, N, Hq + 2 * Hkv, D)
        x[:, :, Hq:] += randn(g, 1, 1, 2 * Hkv, D)
        x = x.to(dt).transpose(1, 2)
        q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    else:
        q, k = randn(g, B, Hq, N, D).to(dt), (randn(g, B, Hkv, N, D) + 3).to(dt)
    w = [1 + 0.3 * randn(g, D) for _ in range(2)] if weights else [None, None]
    inv = (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / max(R, 1))).float()
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda").to(torch.int32)
    pos = {"0": None, "start": ints(0, 200000, B), "each": ints(-50, 5000, B, N), "far": ints(2 ** 30, 2 ** 31 - 1000, B)}[at]
    p = torch.arange(N, device="cuda").expand(B, N)
    if pos is not None:
        p = pos.long() if pos.dim() == 2 else p + pos.long()[:, None]
    n = torch.full((B,), N, device="cuda") if lens is None else torch.tensor(lens, device="cuda")
    live = (torch.arange(N, device="cuda") < n[:, None])[:, None, :, None]
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(pos=pos, lens=ln, eps=1e-5, interleaved=pairs)
    return g, q, k, w, inv, kw, p, live


def check_rope(case, q, k, w, inv, p, live, zq, zk, label):
    import torch
    pairs, D, R = case[6], case[4], case[5]
    th = mo.angles(inv, p)[:, None]
    worst = 0.0
    for x, wt, z in ((q, w[0], zq), (k, w[1], zk)):
        wt = torch.ones(D, dtype=torch.float64, device="cuda") if wt is None else wt.double()
        y, want = mo.norm_rope(x.double(), wt, th, pairs, 1e-5, live)
        t = mo.norm_rope_bound(y, want, R, pairs, p, _lm.unit(x.dtype), live)
        d = (z.double() - want).abs()
        assert bool((d <= t).all()), "%s: off by %.3g of its bound" % (label, float((d / t.clamp_min(1e-300)).max()))
        worst = max(worst, float((d / t.clamp_min(1e-300)).max()))
    say("%s: at %.3f of its bound" % (label, worst))


@pytest.mark.parametrize("case", ROPES)
def test_norm_rope_forward(case):
    import torch
    g, q, k, w, inv, kw, p, live = rope_case(case)
    say("norm_rope %s" % (case,))
    if kw["lens"] is not None:                           # what lies behind is not read
        for x in (q, k):
            x.copy_(torch.where(live, x, math.nan))
    zq, zk = bd.sage_qk_norm_rope_fwd(q, k, *w, inv, **kw)
    torch.cuda.synchronize()
    check_rope(case, q, k, w, inv, p, live, zq, zk, "norm_rope %s" % (case,))
    # strided outputs, and in place
    zs = [torch.full(x.shape[:2] + (x.shape[2] + 1, x.shape[3] + 8), 5.0, dtype=x.dtype, device="cuda") for x in (q, k)]
    bd.sage_qk_norm_rope_fwd(q, k, *w, inv, out=[z[:, :, :-1, :-8] for z in zs], **kw)
    for z, want in zip(zs, (zq, zk)):
        assert torch.equal(z[:, :, :-1, :-8], want) and bool((z[:, :, -1] == 5).all()) and bool((z[..., -8:] == 5).all())
    bd.sage_qk_norm_rope_fwd(q, k, *w, inv, out=(q, k), **kw)
    assert torch.equal(q, zq) and torch.equal(k, zk)


@pytest.mark.parametrize("case", ROPES)
def test_norm_rope_backward(case):
    import torch
    B, Hq, Hkv, N, D, R, pairs = case[:7]
    g, q, k, w, inv, kw, p, live = rope_case(case)
    dq, dk = (randn(g, *x.shape).to(x.dtype) for x in (q, k))
    say("norm_rope backward %s" % (case,))
    if kw["lens"] is not None:
        for x in (q, k, dq, dk):
            x.copy_(torch.where(live, x, math.nan))
    got = bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dq, dk, **kw)
    torch.cuda.synchronize()
    th = mo.angles(inv, p)[:, None]
    for x, wt, dz, gx, gw in ((q, w[0], dq, got[0], got[2]), (k, w[1], dk, got[1], got[3])):
        w64 = torch.ones(D, dtype=torch.float64, device="cuda") if wt is None else wt.double()
        x64, dz64 = torch.where(live, x.double(), 0.0), torch.where(live, dz.double(), 0.0)
        dx, dw, tx, tw = mo.norm_rope_grads(x64, w64, th, pairs, 1e-5, live, dz64, p, _lm.unit(x.dtype))
        d = (gx.double() - torch.where(live, dx, 0.0)).abs()
        say("  dx at %.3f of its bound" % float((d / tx.clamp_min(1e-300)).max()))
        assert bool((d <= tx).all())
        if wt is None:
            assert gw is None
        else:
            say("  dw at %.3f" % float(((gw.double() - dw).abs() / tw).max()))
            assert bool(((gw.double() - dw).abs() <= tw).all())
        # against differences: the slope of sum(z dz) along the gradient itself
        def loss(xx, ww):
            return float((mo.norm_rope(xx, ww, th, pairs, 1e-5, live)[1] * dz64).sum())
        for g_, t_, move in ((gx, tx, lambda h: loss(x64 + h * dx, w64)),) + (
                () if wt is None else ((gw, tw, lambda h: loss(x64, w64 + h * dw)),)):
            d_ = torch.where(live, dx, 0.0) if g_ is gx else dw
            h = 1e-4 / max(1e-300, float(d_.abs().max()))
            near, far = ((move(s) - move(-s)) / (2 * s) for s in (h / 2, h))
            slope = (4 * near - far) / 3                 # the rest is of order h^4
            tol = float((t_ * d_.abs()).sum()) + 1e-6 * abs(slope) + 1e-9
            assert abs(float((g_.double() * d_).sum()) - slope) <= tol
    # the same bits again; in place; into views of one gradient of the projection
    again = bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dq, dk, **kw)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))
    pack = torch.full((B, N, Hq + Hkv + 1, D), 9.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    ws = torch.empty(bd.qk_norm_rope_bwd_workspace_size(B, Hq, Hkv, N, D), dtype=torch.uint8, device="cuda")
    bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dq, dk, workspace=ws, out=(pack[:, :Hq], pack[:, Hq:Hq + Hkv]) + got[2:], **kw)
    assert torch.equal(pack[:, :Hq], got[0]) and torch.equal(pack[:, Hq:Hq + Hkv], got[1]) and bool((pack[:, -1] == 9).all())
    bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dq, dk, out=(dq, dk, None, None), **kw)
    assert torch.equal(dq, got[0]) and torch.equal(dk, got[1])


@pytest.mark.parametrize("dtype,scale", [("fp16", 6e4), ("fp16", 1e-6), ("bf16", 1e18), ("bf16", 1e-30)])
def test_norm_rope_small_and_large_rows(dtype, scale):
    import torch
    g = gen(5)
    dt = getattr(torch, DT[dtype])
    q, k = ((torch.rand((1, 4, 9, 128), generator=g, device="cuda") * scale).to(dt) for _ in range(2))
    inv = torch.ones(64, device="cuda")
    p = torch.arange(9, device="cuda")[None]
    live = torch.ones((1, 1, 9, 1), dtype=torch.bool, device="cuda")
    zq, zk = bd.sage_qk_norm_rope_fwd(q, k, None, None, inv, eps=1e-5)
    check_rope((1, 4, 4, 9, 128, 128, False), q, k, (None, None), inv, p, live, zq, zk, "rows of %g" % scale)


# ---------------------------------------------------------------- the MXFP4 cache
def fp4_cache(g, S, Hkv, page, D, lens, layout="hnd", spare=3, wide=False):
    """A cache with random pages for sequences of these lengths; its tensors, the values they stand for, the table."""
    import torch
    M = max(1, max(-(-max(0, n) // page) for n in lens))
    P = S * M + spare
    c = {}
    for x in "kv":
        c[x + "_cache"] = torch.randint(0, 256, (P, Hkv, page, D // 2), generator=g, device="cuda").to(torch.uint8)
        c[x + "_scale"] = (126 + torch.randint(-6 if wide else -1, 4 if wide else 2, (P, Hkv, page, D // 32), generator=g,
                                               device="cuda")).to(torch.uint8)
        if layout == "nhd":
            c[x + "_cache"] = c[x + "_cache"].transpose(1, 2).contiguous().transpose(1, 2)
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    return c, perm[:S * M].view(S, M).contiguous(), perm[S * M:]


def check_decode(q, c, table, lens, window, sinks, o, lse, label, w0=None, w1=None):
    """(w1: the weights w0 after the call.  Each weight is exp(S - L): S and L are off by e each, the power and the
    logarithm and the sum that L is of by (n + 64) 2^-23 together; G weights and the old sum are added up.)"""
    import torch
    S, Hq, D = q.shape
    Hkv, page = c["k_cache"].shape[1:3]
    G, u = Hq // Hkv, _lm.unit(q.dtype)
    k, v = (mo.fp4_values(c[x + "_cache"], c[x + "_scale"]) for x in "kv")
    tab = table.cpu()
    worst = [0.0, 0.0, 0.0]
    for s in range(S):
        n = max(0, min(int(lens[s]), table.shape[1] * page))
        for h in range(Hkv):
            kr, has = _lm.cache_rows(k, None, tab[s], h, n)
            vr, _ = _lm.cache_rows(v, None, tab[s], h, n)
            hs = slice(h * G, (h + 1) * G)
            r = mo.fp4_decode(q[s, hs].double(), kr, vr, has.to(q.device), window, sinks)
            worst[0] = max(worst[0], float(((o[s, hs].double() - r["o"]).abs() / _lm.o_bound(r, n, u, 2.0 ** -16)).max()))
            dead = r["lse"] == -math.inf
            assert bool((lse[s, hs][dead] == -math.inf).all()), label
            d = torch.where(dead, 0.0, lse[s, hs].double() - r["lse"]).abs()
            worst[1] = max(worst[1], float((d / _lm.lse_bound(r, n)).max()))
            if w1 is not None and n:
                want = w0[s, h, :n].double() + r["p"].sum(0)
                tol = ((2 * r["e"] + (n + 64) * 2.0 ** -23) * r["p"]).sum(0) + (G + 2) * 2.0 ** -24 * want.abs() + 1e-30
                worst[2] = max(worst[2], float(((w1[s, h, :n].double() - want).abs() / tol).max()))
        if w1 is not None:
            assert torch.equal(w1[s, :, n:], w0[s, :, n:]), label
    say("%s: O at %.3f of its bound, L at %.3f, weights at %.3f" % (label, *worst))
    assert max(worst) <= 1, label


DECODES = [
    # Hq, Hkv, page, D, lens, dtype, layout, window, sinks
    (1, 1, 16, 128, [1], "bf16", "hnd", None, 0),
    (1, 1, 16, 64, [1], "bf16", "hnd", None, 0),
    (8, 2, 16, 64, [77], "fp16", "hnd", None, 0),
    (8, 2, 16, 64, [70], "bf16", "nhd", None, 0),
    (16, 2, 32, 128, [63, 64, 65], "bf16", "hnd", None, 0),
    (32, 2, 1, 128, [130], "bf16", "hnd", None, 0),
    (8, 8, 1, 128, [40, 3], "bf16", "hnd", None, 0),
    (4, 1, 24, 128, [100, 0, 25], "fp16", "nhd", None, 0),
    (32, 8, 64, 128, [1700, 1, 512, 1025, 1024], "bf16", "hnd", None, 0),
    (20, 1, 32, 128, [300, 1900], "fp16", "nhd", None, 0),
    (64, 2, 128, 64, [1000, 1330], "bf16", "hnd", None, 0),
    (12, 2, 16, 128, [1650, 31, 32, 33, 640], "fp16", "hnd", None, 0),
    (6, 2, 256, 128, [3000], "bf16", "nhd", 128, 4),
    (8, 2, 32, 128, [1500, 64, 9], "bf16", "hnd", 100, 4),
    (8, 8, 48, 64, [1200, 600], "fp16", "hnd", 1, 0),
    (4, 4, 64, 128, [1300, 0, 0, 640], "bf16", "hnd", 257, 70),
    (14, 2, 16, 64, [1900, 8], "fp16", "hnd", 64, 1),
    (3, 3, 16, 128, [5000, 4999], "bf16", "hnd", 4000, 100),
]


@pytest.mark.parametrize("case", DECODES)
def test_paged_decode_fp4(case):
    import torch
    Hq, Hkv, page, D, lens, dtype, layout, window, sinks = case
    g = gen(100 + sum(lens) + D)
    S = len(lens)
    c, table, _ = fp4_cache(g, S, Hkv, page, D, lens, layout)
    q = (0.5 * randn(g, S, Hq, D)).to(getattr(torch, DT[dtype]))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    say("decode fp4 %s" % (case,))
    args = (c["k_cache"], c["v_cache"], table, ln)
    kw = dict(window=window, sinks=sinks, k_scale=c["k_scale"], v_scale=c["v_scale"])
    o, lse = bd.sage_attn_paged_decode(q, *args, **kw)
    torch.cuda.synchronize()
    check_decode(q, c, table, lens, window, sinks, o, lse, "decode fp4 %s" % (case,))
    # the same bits again, without L, from a strided q
    pad = torch.zeros((S, Hq + 3, D + 8), dtype=q.dtype, device="cuda")
    pad[:, :Hq, :D] = q
    o2, none = bd.sage_attn_paged_decode(pad[:, :Hq, :D], *args, lse=False, **kw)
    assert torch.equal(o, o2) and none is None


@pytest.mark.parametrize("case", DECODES)
def test_paged_decode_fp4_weights(case):
    """The weights are added up as they are over other caches; the rest of the answer stays."""
    import torch
    Hq, Hkv, page, D, lens, dtype, layout, window, sinks = case
    g = gen(200 + sum(lens) + D)
    S = len(lens)
    c, table, _ = fp4_cache(g, S, Hkv, page, D, lens, layout)
    q = (0.5 * randn(g, S, Hq, D)).to(getattr(torch, DT[dtype]))
    if S > 1:
        table[-1, 0] = -1                                # a hole
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    say("weights fp4 %s" % (case,))
    args = (c["k_cache"], c["v_cache"], table, ln)
    kw = dict(window=window, sinks=sinks, k_scale=c["k_scale"], v_scale=c["v_scale"])
    w0 = torch.rand((S, Hkv, table.shape[1] * page + 5), generator=g, device="cuda")
    w1, w2, w3 = w0.clone(), w0.clone(), w0.clone()
    o, lse = bd.sage_attn_paged_decode(q, *args, weights=w1, **kw)
    torch.cuda.synchronize()
    check_decode(q, c, table, lens, window, sinks, o, lse, "weights fp4 %s" % (case,), w0, w1)
    o2, lse2 = bd.sage_attn_paged_decode(q, *args, weights=w2, **kw)
    o3, lse3 = bd.sage_attn_paged_decode(q, *args, **kw)
    assert torch.equal(w1, w2)
    for x, y in ((o2, lse2), (o3, lse3)):
        assert torch.equal(o, x) and torch.equal(lse, y)
    bd.sage_attn_paged_decode(q, *args, lse=False, weights=w3, **kw)
    assert torch.equal(w1, w3)


EVICTS = [
    # Hkv, page, D, lens, budget, first, last, layout
    (1, 16, 64, [1], 1, 0, 0, "hnd"),
    (2, 16, 64, [100, 40, 0, 41], 40, 4, 8, "hnd"),
    (2, 24, 128, [2500, 999, 1000, 1001], 1000, 16, 300, "nhd"),
    (3, 1, 64, [77, 30], 20, 20, 0, "nhd"),
    (2, 64, 128, [700], 699, 0, 0, "hnd"),
    (1, 128, 128, [20000], 1, 0, 0, "hnd"),
    (1, 32, 64, [20000], 300, 100, 200, "hnd"),
]


@pytest.mark.parametrize("case", EVICTS)
def test_evict_fp4(case):
    """The kept tokens by their definition; their codes and scales bit for bit; nothing else of the cache changes."""
    import torch
    Hkv, page, D, lens, budget, first, last, layout = case
    g = gen(sum(lens) + budget)
    S, M2 = len(lens), -(-budget // page)
    c, table, spare = fp4_cache(g, S, Hkv, page, D, lens, layout, spare=S * M2 + 2, wide=True)
    new_table = spare[:S * M2].view(S, M2).contiguous()
    w = torch.exp(3 * randn(g, S, Hkv, table.shape[1] * page + 7) - 6)
    if D == 64:
        w = torch.round(w * 4) / 4                       # ties
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = {x: t.clone() for x, t in c.items()}
    say("evict fp4 %s" % (case,))
    nl, nw, kept = bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, w, new_table, budget, first, last, k_scale=c["k_scale"],
                                    v_scale=c["v_scale"])
    torch.cuda.synchronize()
    assert nl.tolist() == [min(n, budget) for n in lens]
    wc, tc, ntc = w.cpu().numpy(), table.cpu().numpy(), new_table.cpu().numpy()
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).long().cuda()
    for s, n in enumerate(lens):
        for h in range(Hkv):
            keep = _lm.kept_tokens(wc[s, h, :n], n, budget, first, last)
            m = len(keep)
            got, j = kept[s, h].cpu().numpy(), np.arange(m)
            assert np.array_equal(got[:m], keep) and (got[m:] == -1).all(), (s, h)
            assert torch.equal(nw[s, h, :m], w[s, h][dev(keep)]) and not bool(nw[s, h, m:].any())
            for x in want:
                want[x][dev(ntc[s, j // page]), h, dev(j % page)] = want[x][dev(tc[s, keep // page]), h, dev(keep % page)]
    for x in c:
        assert torch.equal(c[x], want[x]), x


@pytest.mark.parametrize("D", [64, 128])
def test_tokens_weights_and_eviction_over_fp4(D):
    """Prompts stored, tokens one at a time by a captured graph that adds up the weights, an eviction by these, and tokens
    over what is left: every answer is the attention over the rows that the cache holds."""
    import torch
    g = gen(78)
    S, Hq, Hkv, N, T, page = 3, 8, 2, 90, 8, 16
    lens0 = [90, 41, 7]
    M = -(-(N + T) // page)
    c, table, spare = fp4_cache(g, S, Hkv, page, D, [M * page] * S, spare=3 * S)
    kw = dict(k_scale=c["k_scale"], v_scale=c["v_scale"])
    i32 = dict(dtype=torch.int32, device="cuda")
    w = torch.full((S, Hkv, M * page), 9.0, device="cuda")
    lens = torch.tensor(lens0, **i32)
    k, v = (randn(g, S, Hkv, N, D).to(torch.bfloat16) for _ in "kv")
    bd.sage_kv_append(k, v, c["k_cache"], c["v_cache"], table, torch.zeros(S, **i32), lens, weights=w, **kw)
    assert all(bool((w[s, :, :n] == 0).all()) and bool((w[s, :, n:] == 9).all()) for s, n in enumerate(lens0))
    q, kt, vt = torch.zeros((S, Hq, D), dtype=torch.bfloat16, device="cuda"), *(torch.zeros((S, Hkv, 1, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")

    def step(c, lens, w):
        sc = dict(k_scale=c["k_scale"], v_scale=c["v_scale"])
        bd.sage_kv_append(kt, vt, c["k_cache"], c["v_cache"], table, lens, weights=w, **sc)
        lens += 1
        return bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, lens, window=64, sinks=4, weights=w, **sc)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step({x: t.clone() for x, t in c.items()}, lens.clone(), w.clone())
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step(c, lens, w)
    for t in range(T):
        q.copy_(0.5 * randn(g, S, Hq, D)), kt.copy_(randn(g, S, Hkv, 1, D)), vt.copy_(randn(g, S, Hkv, 1, D))
        eager = ({x: t.clone() for x, t in c.items()}, lens.clone(), w.clone())
        w0 = w.clone()
        for s in range(S):
            w0[s, :, lens[s]] = 0                        # a new token begins with none
        graph.replay()
        want = step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(w, eager[2]) and torch.equal(lens, eager[1])
        assert all(torch.equal(c[x], eager[0][x]) for x in c)
        check_decode(q, c, table, lens.tolist(), 64, 4, o, lse, "token %d" % t, w0, w)
    new_table = spare[:3 * S].view(S, 3).contiguous()
    nl, nw, kept = bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, lens, w, new_table, 40, 4, 16, **kw)
    assert nl.tolist() == [min(n + T, 40) for n in lens0]
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], new_table, nl, **kw)
    torch.cuda.synchronize()
    check_decode(q, c, new_table, nl.tolist(), None, 0, o, lse, "after the eviction")
    for s in range(S):
        m = int(nl[s])
        for h in range(Hkv):
            i = kept[s, h, :m].long()
            j = torch.arange(m, device="cuda")
            for x in c:
                assert torch.equal(c[x][new_table[s][j // page].long(), h, j % page], c[x][table[s][i // page].long(), h, i % page]), x
            assert torch.equal(nw[s, h, :m], w[s, h][i])


@pytest.mark.parametrize("D", [64, 128])
def test_paged_decode_fp4_layouts(D):
    """K and V of differing strides, and pages of 16-token multiples or not, give the same; a captured call follows
    the lengths and tables."""
    import torch
    g = gen(31)
    lens = [1500, 33, 700]
    c, table, _ = fp4_cache(g, 3, 2, 48, D, lens)
    q = (0.5 * randn(g, 3, 10, D)).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(window=900, sinks=3, k_scale=c["k_scale"], v_scale=c["v_scale"])
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, **kw)
    check_decode(q, c, table, lens, 900, 3, o, lse, "pages of 48, D %d" % D)
    other = c["v_cache"].transpose(1, 2).contiguous().transpose(1, 2)
    again = bd.sage_attn_paged_decode(q, c["k_cache"], other, table, ln, **kw)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    # pages of 24: each of the 48 cut into two
    cut = {x: t.unflatten(2, (2, 24)).transpose(1, 2).flatten(0, 1).contiguous() for x, t in c.items()}
    halves = torch.stack([2 * table, 2 * table + 1], -1).flatten(1).contiguous()
    again = bd.sage_attn_paged_decode(q, cut["k_cache"], cut["v_cache"], halves, ln, window=900, sinks=3, k_scale=cut["k_scale"],
                                      v_scale=cut["v_scale"])
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, **kw)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, **kw)
    for new in ([1500, 33, 700], [0, 1536, 48], [64, 65, 1000], [1, 0, 0]):
        ln.copy_(torch.tensor(new, dtype=torch.int32))
        table.copy_(table.flip(0))
        graph.replay()
        want = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, **kw)
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_paged_decode_fp4_wide_scales_and_large_q(D, dtype):
    """Blocks of differing scales, channels of q that differ by 2^10 and more in size, scores of many sizes."""
    import torch
    g = gen(9)
    lens = [900, 130]
    c, table, _ = fp4_cache(g, 2, 2, 16, D, lens, wide=True)
    q = (0.2 * randn(g, 2, 8, D) * torch.exp2(torch.randint(-14, 3, (1, 1, D), generator=g, device="cuda").float()))
    q = q.to(getattr(torch, DT[dtype]))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, k_scale=c["k_scale"], v_scale=c["v_scale"])
    check_decode(q, c, table, lens, None, 0, o, lse, "wide scales, D %d, %s" % (D, dtype))


@pytest.mark.parametrize("S,Hkv", [(64, 2), (65, 1), (300, 1)])
def test_paged_decode_fp4_many_ragged_sequences(S, Hkv):
    import torch
    g = gen(3)
    page, D = 16, 64
    lens = [int(x) for x in np.random.default_rng(4).integers(0, 1500, S)]
    lens[0], lens[62], lens[-1] = 0, 1499, 0
    lens[1:3] = [0, 0]
    c, table, _ = fp4_cache(g, S, Hkv, page, D, lens)
    q = (0.5 * randn(g, S, 4 * Hkv, D)).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, k_scale=c["k_scale"], v_scale=c["v_scale"])
    torch.cuda.synchronize()
    pick = sorted({i % S for i in (0, 1, 2, 3, 31, 62, 63, S // 2, -3, -2, -1)})
    sub = torch.tensor(pick, device="cuda")
    check_decode(q[sub], c, table[sub], [lens[i] for i in pick], None, 0, o[sub], lse[sub], "%d sequences" % S)


def test_paged_decode_fp4_ignores_what_it_does_not_see():
    """Rows behind the ends, outside the window and on pages that the cache does not have: scales that stand for
    NaN (byte 255) there change nothing, and a NaN in q stays in its head."""
    import torch
    g = gen(12)
    lens, page, D = [1500, 70, 0], 16, 128
    c, table, spare = fp4_cache(g, 3, 2, page, D, lens)
    q = (0.5 * randn(g, 3, 8, D)).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table[0, 3], table[0, 90], table[1, 1] = -1, c["k_cache"].shape[0], 2 ** 31 - 1
    kw = dict(window=200, sinks=70)
    run = lambda: bd.sage_attn_paged_decode(q, c["k_cache"], c["v_cache"], table, ln, k_scale=c["k_scale"], v_scale=c["v_scale"], **kw)
    o, lse = run()
    check_decode(q, c, table, lens, 200, 70, o, lse, "holes")
    seen = torch.zeros(c["k_cache"].shape[:1] + (page,), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for j in range(n):
            if (j >= n - 200 or j < 70) and 0 <= int(table[s, j // page]) < len(seen):
                seen[int(table[s, j // page]), j % page] = True
    for x in "kv":
        c[x + "_scale"] = torch.where(seen[:, None, :, None], c[x + "_scale"], 255).to(torch.uint8)
    o2, lse2 = run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    q[0, 5, 100] = math.nan
    o2, lse2 = run()
    assert bool(o2[0, 5].isnan().all()) and bool(lse2[0, 5].isnan())
    o2[0, 5], lse2[0, 5] = o[0, 5], lse[0, 5]
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def new_tokens(g, S, Hkv, N, D, dtype, kind):
    """Rows of new tokens: normal ones, or blocks of zeros, ties, and sizes at the type's ends."""
    import torch
    x = randn(g, S, Hkv, N, D) * torch.exp2(torch.randint(-8, 8, (S, Hkv, N, D // 32), generator=g, device="cuda").float()).repeat_interleave(32, -1)
    if kind == "edges":
        at = torch.randint(0, 6, (S, Hkv, N, D // 32), generator=g, device="cuda").repeat_interleave(32, -1)
        ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, 0.0, -0.0], device="cuda")
        pick = ties[torch.randint(0, len(ties), x.shape, generator=g, device="cuda")]
        small, large = (2.0 ** -133, 2.0 ** 126) if dtype == "bf16" else (2.0 ** -24, 2.0 ** 14)
        r = torch.randint(1, 4, x.shape, generator=g, device="cuda").float()
        x = torch.where(at == 0, 0.0, torch.where(at == 1, pick, torch.where(at == 2, small * r, torch.where(at == 3, large * r.clamp(max=1.5), x))))
        x = torch.where(at == 4, x.sign() * 2.0 ** -126 if dtype == "bf16" else x, x)
    return x.to(getattr(torch, DT[dtype]))


@pytest.mark.parametrize("kind", ["normal", "edges"])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,D,page,N", [("bf16", 128, 16, 1), ("fp16", 64, 24, 50), ("bf16", 64, 1, 7), ("fp16", 128, 64, 131)])
def test_append_fp4(dtype, D, page, N, layout, kind):
    """Codes and scales bit for bit, everything else as it was."""
    import torch
    g = gen(N + D)
    S, Hkv = 3, 2
    c, table, _ = fp4_cache(g, S, Hkv, page, D, [N + 30] * S, layout)
    table[2, 0] = -5                                     # no page: not stored
    k, v = (new_tokens(g, S, Hkv, N, D, dtype, kind) for _ in range(2))
    pos, counts = torch.tensor([3, 0, 7], dtype=torch.int32, device="cuda"), torch.tensor([N, N - 1, N + 9], dtype=torch.int32, device="cuda")
    want = {x: t.clone() for x, t in c.items()}
    for s in range(S):
        for t in range(min(int(counts[s]), N)):
            at = int(pos[s]) + t
            pid = int(table[s, at // page])
            if not 0 <= pid < len(c["k_cache"]):
                continue
            for x, rows in (("k", k), ("v", v)):
                codes, sc = mo.fp4_rows(rows[s, :, t].double().cpu().numpy())
                want[x + "_cache"][pid, :, at % page] = torch.from_numpy(codes).cuda()
                want[x + "_scale"][pid, :, at % page] = torch.from_numpy(sc).cuda()
    bd.sage_kv_append(k, v, c["k_cache"], c["v_cache"], table, pos, counts=counts, k_scale=c["k_scale"], v_scale=c["v_scale"])
    torch.cuda.synchronize()
    for x in c:
        assert torch.equal(c[x], want[x]), x


@pytest.mark.parametrize("kind", ["16", "int8", "fp4"])
@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("dtype,D,page,N", [("bf16", 128, 16, 1), ("fp16", 64, 24, 50), ("fp16", 128, 64, 131), ("bf16", 64, 1, 7)])
def test_append_by_slots_equals_append_by_tables(dtype, D, page, N, flat, kind):
    import torch
    g = gen(N + D)
    S, Hkv = 3, 5
    dt = getattr(torch, DT[dtype])
    c, table, _ = fp4_cache(g, S, Hkv, page, D, [N + 30] * S)
    P = len(c["k_cache"])
    if kind == "16":
        c = {x: (torch.zeros((P, Hkv, page, D), dtype=dt, device="cuda") if "cache" in x else None) for x in c}
    if kind == "int8":
        c = {x: torch.zeros((P, Hkv, page, D), dtype=torch.int8, device="cuda") if "cache" in x
             else torch.zeros((P, Hkv, page), device="cuda") for x in c}
    other = {x: None if t is None else t.clone() for x, t in c.items()}
    k, v = (randn(g, S, Hkv, N, D).to(dt) for _ in range(2))
    pos, counts = torch.tensor([3, 0, 7], dtype=torch.int32, device="cuda"), torch.tensor([N, N - 1, N // 2], dtype=torch.int32, device="cuda")
    bd.sage_kv_append(k, v, c["k_cache"], c["v_cache"], table, pos, counts=counts, k_scale=c["k_scale"], v_scale=c["v_scale"])
    t = torch.arange(N, device="cuda")
    at = pos.long()[:, None] + t
    slots = table.long().gather(1, at // page) * page + at % page
    slots = torch.where(t < counts[:, None], slots, torch.tensor([[-1], [P * page], [2 ** 40]], device="cuda"))
    if flat:
        slots = slots.flatten()[None].contiguous()
        k, v = (x.transpose(1, 2).flatten(0, 1).transpose(0, 1)[None] for x in (k, v))       # [1, Hkv, S N, D] of [S N, Hkv, D]
    bd.sage_kv_append_slots(k, v, other["k_cache"], other["v_cache"], slots.contiguous(), k_scale=other["k_scale"], v_scale=other["v_scale"])
    torch.cuda.synchronize()
    for x in c:
        assert c[x] is None or torch.equal(c[x], other[x]), x


@pytest.mark.parametrize("gib", [1, 3, 4])
def test_fp4_caches_beyond_32_bit_offsets(gib):
    """Pages behind 2^30, 2^31 and 2^32 bytes of the cache: stored and read as in a small one."""
    import torch
    g = gen(51)
    S, Hkv, page, D, lens = 2, 16, 256, 128, [1700, 513]
    c, table, _ = fp4_cache(g, S, Hkv, page, D, lens)
    q = (0.5 * randn(g, S, 32, D)).to(torch.bfloat16)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kn, vn = (randn(g, S, Hkv, 1, D).to(torch.bfloat16) for _ in range(2))
    P, n = len(c["k_cache"]), gib * 2 ** 30 // (Hkv * page * D // 2)
    big = {}
    for x, t in c.items():                               # the same pages, n places further on
        big[x] = torch.zeros((n + P,) + tuple(t.shape[1:]), dtype=torch.uint8, device="cuda")
        big[x][n:] = t
    outs = []
    for cc, off in ((c, 0), (big, n)):
        kw = dict(k_scale=cc["k_scale"], v_scale=cc["v_scale"])
        bd.sage_kv_append(kn, vn, cc["k_cache"], cc["v_cache"], table + off, ln - 1, **kw)
        slots = ((table[:, :1] + off).long() * page + 5).contiguous()
        bd.sage_kv_append_slots(vn, kn, cc["k_cache"], cc["v_cache"], slots, **kw)
        outs.append(bd.sage_attn_paged_decode(q, cc["k_cache"], cc["v_cache"], table + off, ln, **kw))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert all(torch.equal(big[x][n:], c[x]) for x in c)


def test_append_by_slots_past_32_bits():
    """Slots past 2^31: pages of few bytes."""
    import torch
    g = gen(52)
    k1, v1 = (torch.zeros((2 ** 21 + 2, 1, 1024, 32), dtype=torch.uint8, device="cuda") for _ in range(2))
    s1, s2 = (torch.zeros((2 ** 21 + 2, 1, 1024, 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    x = randn(g, 1, 1, 2, 64).to(torch.bfloat16)
    slots = torch.tensor([[2 ** 31 + 1500, 3]], device="cuda")
    bd.sage_kv_append_slots(x, x, k1, v1, slots, k_scale=s1, v_scale=s2)
    codes, sc = mo.fp4_rows(x[0, 0].double().cpu().numpy())
    assert (k1[2 ** 21 + 1, 0, 476].cpu().numpy() == codes[0]).all() and (k1[0, 0, 3].cpu().numpy() == codes[1]).all()
    assert (s2[2 ** 21 + 1, 0, 476].cpu().numpy() == sc[0]).all() and int(s1.count_nonzero()) == 4


# ---------------------------------------------------------------- page tables
def requests(rng, S, page, M, N, ended=0.2, pages=None, n_free=None):
    """A consistent pool: tables whose pages are distinct, the rest on the stack."""
    had = rng.integers(0, M * page + 1, S) * (rng.random(S) < 0.8)
    counts = rng.integers(0, N + 1, S)
    counts[rng.random(S) < ended] = -1
    held = -(-had // page)
    pages = int(held.sum()) + S * 2 + 5 if pages is None else pages
    ids = rng.permutation(pages).astype(np.int32)
    table = np.full((S, M), -1, np.int32)
    i = 0
    for s in range(S):
        table[s, :held[s]] = ids[i:i + held[s]]
        i += int(held[s])
    free = np.concatenate([ids[i:], np.full(i, -7, np.int32)])
    return table, had.astype(np.int32), counts.astype(np.int32), free, np.array([pages - i if n_free is None else n_free], np.int32)


PLANS = [
    # S, page, M, N, ended, n_free, T
    (1, 16, 4, 3, 0.0, None, 8),
    (1, 1, 1, 1, 1.0, None, 1),
    (7, 24, 9, 50, 0.2, None, 400),
    (256, 16, 20, 1, 0.1, None, 256),
    (300, 16, 20, 40, 0.2, 30, 12000),
    (1023, 8, 5, 9, 0.3, None, 4096),
    (1025, 8, 5, 9, 0.3, None, 4097),
    (2500, 4, 6, 20, 0.2, None, 9000),
    (5000, 64, 3, 30, 0.9, 0, 70000),
    (40, 128, 3, 100, 0.0, 5, 60),
    (3, 2, 2000, 3000, 0.0, None, 9000),
]


@pytest.mark.parametrize("case", PLANS)
def test_plan(case):
    import torch
    torch_dev()
    S, page, M, N, ended, n_free, T = case
    rng = np.random.default_rng(S + T)
    say("plan %s" % (case,))
    for rep in range(3):
        args = requests(rng, S, page, M, N, ended, n_free=n_free)
        want = mo.plan(*args, page, T)
        dev = [torch.from_numpy(x.copy()).cuda() for x in args]
        out = bd.sage_kv_plan(*dev, page, T)
        torch.cuda.synchronize()
        got = (dev[0], dev[1], dev[3], dev[4]) + tuple(out)
        names = ("table", "lens", "free", "n_free", "granted", "starts", "pos", "slots")
        for a, b, what in zip(got, want, names):
            assert (a.cpu().numpy() == b).all(), what
        assert torch.equal(dev[2].cpu(), torch.from_numpy(args[2]))


def test_plan_odd_states():
    """Lengths and stack heights out of range count as their nearest ends; a full stack drops what is returned; more
    tokens than a row holds are not granted, and hold nobody up."""
    import torch
    torch_dev()
    table = np.arange(24, dtype=np.int32).reshape(4, 6)
    lens = np.array([-5, 1000, 24, 0], np.int32)
    for counts in ([3, 1, -1, 2 ** 31 - 1], [-1, -1, -1, -1], [0, 0, 0, 0], [25, 25, 25, 24], [24, -1, 0, 24]):
        for n_free, T in ((-3, 50), (5, 50), (99, 50), (8, 5000), (8, 24)):
            args = (table, lens, np.array(counts, np.int32), np.arange(100, 110, dtype=np.int32), np.array([n_free], np.int32))
            want = mo.plan(*args, 4, T)
            dev = [torch.from_numpy(x.copy()).cuda() for x in args]
            got = (dev[0], dev[1], dev[3], dev[4]) + tuple(bd.sage_kv_plan(*dev, 4, T))
            for a, b in zip(got, want):
                assert (got is not None) and (a.cpu().numpy() == b).all(), (counts, n_free, T)


def test_binding_refuses_mismatched_tensors():
    """Every check of the binding that a bare pointer cannot carry; nothing is launched, nothing changes."""
    import torch
    g = gen(1)
    q, k = randn(g, 2, 8, 5, 64).to(torch.bfloat16), randn(g, 2, 2, 5, 64).to(torch.bfloat16)
    w, inv, z = torch.ones(64, device="cuda"), torch.ones(32, device="cuda"), torch.zeros
    i32 = dict(dtype=torch.int32, device="cuda")
    fwd = lambda q=q, k=k, qw=w, kw=w, inv=inv, **a: bd.sage_qk_norm_rope_fwd(q, k, qw, kw, inv, **a)
    for bad in (dict(k=k[:, :, :4]), dict(k=k.half()), dict(k=randn(g, 2, 3, 5, 64).to(torch.bfloat16)), dict(qw=w[:32]), dict(kw=w.half()),
                dict(qw=w.cpu()), dict(inv=torch.ones(33, device="cuda")), dict(inv=torch.ones(30, device="cuda")), dict(inv=torch.ones(36, device="cuda")),
                dict(pos=z(2, 4, **i32)), dict(pos=z(3, **i32)), dict(pos=z(2, dtype=torch.int64, device="cuda")), dict(lens=z(3, **i32)), dict(eps=0.0),
                dict(eps=2.0), dict(q=q.transpose(-1, -2).contiguous().transpose(-1, -2)), dict(out=(q, k.half())), dict(out=(q[:, :4], k))):
        with pytest.raises(ValueError):
            fwd(**bad)
    bwd = lambda dq=q, dk=k, **a: bd.sage_qk_norm_rope_bwd(q, k, w, w, inv, dq, dk, **a)
    for bad in (dict(dq=q[:1]), dict(dk=k.float()), dict(out=(q, k, w[:3], w)), dict(out=(q, q, w, w)), dict(workspace=z(10, device="cuda"))):
        with pytest.raises(ValueError):
            bwd(**bad)
    with pytest.raises(bd.SageError):
        bwd(workspace=z(256, dtype=torch.uint8, device="cuda"))
    c, table, _ = fp4_cache(g, 2, 2, 16, 64, [40, 40])
    ln, slots = torch.full((2,), 40, **i32), z((2, 5), dtype=torch.int64, device="cuda")
    before = {x: t.clone() for x, t in c.items()}
    sc = dict(k_scale=c["k_scale"], v_scale=c["v_scale"])
    put = lambda k=k, v=k, kc=c["k_cache"], vc=c["v_cache"], s=slots, **a: bd.sage_kv_append_slots(k, v, kc, vc, s, **(a or sc))
    short = dict(k_scale=c["k_scale"][..., :1].contiguous(), v_scale=c["v_scale"])
    for bad in (dict(k=k[:, :1]), dict(v=k[:1]), dict(s=slots[:1]), dict(s=slots.int()), dict(kc=c["k_cache"][..., :16]), dict(vc=c["v_cache"].to(torch.int8)),
                dict(k_scale=None, v_scale=c["v_scale"]), short, dict(k_scale=c["k_scale"].float(), v_scale=c["v_scale"].float())):
        with pytest.raises(ValueError):
            put(**bad)
    one = q[:, :, 0]
    for call in (lambda: bd.sage_attn_paged_decode(one, c["k_cache"], c["v_cache"], table, ln, weights=z((2, 2, 47), device="cuda"), **sc),
                 lambda: bd.sage_attn_paged_decode(one[..., :32], c["k_cache"], c["v_cache"], table, ln, **sc),
                 lambda: bd.sage_attn_paged_decode(one, c["k_cache"], c["v_cache"], table, ln),
                 lambda: bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, z((2, 1, 64), device="cuda"), table.clone(), 16, **sc),
                 lambda: bd.sage_kv_evict(c["k_cache"], c["v_cache"], table, ln, z((2, 2, 64), device="cuda"), table.clone(), 16)):
        with pytest.raises(ValueError):
            call()
    counts, free, n = torch.ones(2, **i32), z(8, **i32), z(1, **i32)
    for bad in ((table.long(), ln, counts, free, n, 16, 8), (table, ln[:1], counts, free, n, 16, 8), (table, ln, counts.float(), free, n, 16, 8),
                (table, ln, counts, free.long(), n, 16, 8), (table, ln, counts, free, z(2, **i32), 16, 8), (table, ln, counts, free, n, 0, 8),
                (table, ln, counts, free, n, 16, 0), (table, ln, counts, free[:0], n, 16, 8)):
        with pytest.raises(ValueError):
            bd.sage_kv_plan(*bad)
    with pytest.raises(ValueError):
        bd.sage_kv_plan(table, ln, counts, free, n, 16, 8, out=(counts, counts, counts, counts))
    torch.cuda.synchronize()
    assert all(torch.equal(c[x], before[x]) for x in c)


# ---------------------------------------------------------------- together
def step_of(st, kind):
    """One step of a batch that generates: pages and slots, norms and rotation, storing, attention."""
    granted, starts, pos, slots = bd.sage_kv_plan(st["table"], st["lens"], st["counts"], st["free"], st["n_free"], st["page"], st["T"])
    q, k, v = st["q"], st["k"], st["v"]
    zq, zk = bd.sage_qk_norm_rope_fwd(q, k, st["wq"], st["wk"], st["inv"], pos=pos[None])
    bd.sage_kv_append_slots(zk, v, st["k_cache"], st["v_cache"], slots[None], k_scale=st["k_scale"], v_scale=st["v_scale"])
    # token i belongs to request i, as every one brings one
    o, lse = bd.sage_attn_paged_decode(zq[0].transpose(0, 1), st["k_cache"], st["v_cache"], st["table"], st["lens"],
                                       k_scale=st["k_scale"], v_scale=st["v_scale"])
    return granted, starts, pos, slots, zq, zk, o, lse


@pytest.mark.parametrize("kind", ["16", "int8", "fp4"])
def test_steps_of_a_batch_captured(kind):
    """Requests that generate, step by step: a captured graph of the four calls, replayed over the state that it
    changes, gives what eager calls give, and the attention is that of the tokens stored so far."""
    import torch
    g = gen(77)
    S, Hq, Hkv, D, page, M = 5, 8, 2, 64, 16, 8
    dt = torch.bfloat16

    def state():
        x = torch.Generator(device="cuda").manual_seed(5)
        P = S * M
        shape = (P, Hkv, page, D // 2 if kind == "fp4" else D)
        ct = {"16": dt, "int8": torch.int8, "fp4": torch.uint8}[kind]
        st = dict(k_cache=torch.zeros(shape, dtype=ct, device="cuda"), v_cache=torch.zeros(shape, dtype=ct, device="cuda"),
                  k_scale=None, v_scale=None, page=page, T=S, table=torch.full((S, M), -1, dtype=torch.int32, device="cuda"),
                  lens=torch.zeros(S, dtype=torch.int32, device="cuda"), counts=torch.ones(S, dtype=torch.int32, device="cuda"),
                  free=torch.randperm(P, generator=x, device="cuda").to(torch.int32), n_free=torch.full((1,), P, dtype=torch.int32, device="cuda"),
                  q=torch.zeros((1, Hq, S, D), dtype=dt, device="cuda"), k=torch.zeros((1, Hkv, S, D), dtype=dt, device="cuda"),
                  v=torch.zeros((1, Hkv, S, D), dtype=dt, device="cuda"), wq=torch.rand(D, generator=x, device="cuda") + 0.5,
                  wk=torch.rand(D, generator=x, device="cuda") + 0.5,
                  inv=(10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float())
        if kind != "16":
            s = (P, Hkv, page) if kind == "int8" else (P, Hkv, page, D // 32)
            sd = torch.float32 if kind == "int8" else torch.uint8
            st.update(k_scale=torch.zeros(s, dtype=sd, device="cuda"), v_scale=torch.zeros(s, dtype=sd, device="cuda"))
        return st

    eager, replayed = state(), state()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step_of(state(), kind)                           # (warms the library up, on another state)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step_of(replayed, kind)
    history = [[] for _ in range(S)]
    for it in range(40):
        q, k, v = (randn(g, *eager[x].shape).to(dt) for x in "qkv")
        counts = [1] * S
        if it == 25:
            counts[2] = -1                               # request 2 ends, and another takes its place
        for st in (eager, replayed):
            st["q"].copy_(q), st["k"].copy_(k), st["v"].copy_(v)
            st["counts"].copy_(torch.tensor(counts, dtype=torch.int32))
        want = step_of(eager, kind)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), it
        for x in ("table", "lens", "free", "n_free", "k_cache", "v_cache", "k_scale", "v_scale"):
            assert eager[x] is None or torch.equal(eager[x], replayed[x]), (it, x)
        row = 0
        for s in range(S):
            if counts[s] < 0:
                history[s] = []
                continue
            history[s].append((want[5][0, :, row].double(), v[0, :, row].double()))
            row += 1
        assert eager["lens"].tolist() == [len(h) for h in history]
        if it in (0, 15, 24) and kind == "16":           # against attention over what was stored
            u = _lm.unit(dt)
            for s in range(S):
                for h in range(Hkv):
                    kr, vr = (torch.stack([t[j][h] for t in history[s]]) for j in range(2))
                    hs = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
                    r = _lm.decode_attention(want[4][0, hs, s].double(), kr, vr, torch.ones(len(kr), dtype=torch.bool, device="cuda"), None, 0)
                    r["e"] = r["e"] * 1.1
                    assert bool(((want[6][s, hs].double() - r["o"]).abs() <= _lm.o_bound(r, len(kr), u, u * u)).all())


def test_training_step_captured_with_window_attention():
    """Norm and rotation, window attention, and both backwards, captured and replayed on new inputs, while eager
    results of the same tensors live; every replay as the eager calls."""
    import torch
    g = gen(8)
    B, Hq, Hkv, N, D = 2, 8, 2, 200, 128
    dt = torch.bfloat16
    qkv = randn(g, B, N, Hq + 2 * Hkv, D).to(dt)
    x = qkv.transpose(1, 2)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    dout, w = randn(g, B, Hq, N, D).to(dt), [1 + 0.1 * randn(g, D) for _ in range(2)]
    inv = (10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float()
    lens = torch.tensor([N, 77], dtype=torch.int32, device="cuda")

    def step():
        zq, zk = bd.sage_qk_norm_rope_fwd(q, k, *w, inv, lens=lens)
        o, lse = bd.sage_attn_window_fwd(zq, zk, v, window=64, sinks=4, lens=lens)
        dzq, dzk, dv = bd.sage_attn_window_bwd(zq, zk, v, o, lse, dout, window=64, sinks=4, lens=lens)
        return (o, lse, dv) + tuple(bd.sage_qk_norm_rope_bwd(q, k, *w, inv, dzq, dzk, lens=lens))

    alive = step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        qkv.copy_(randn(g, *qkv.shape))
        dout.copy_(randn(g, *dout.shape))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert not torch.equal(alive[0], want[0])


def test_norm_rope_beyond_2_31_elements():
    """Tensors and strides past 2^31 elements: as the same rows in a small one."""
    import torch
    g = gen(61)
    N, D = 3, 128
    w, inv = 1 + 0.1 * randn(g, D), torch.rand(64, generator=g, device="cuda")
    big = torch.zeros((2 ** 31 // D + 64, D), dtype=torch.bfloat16, device="cuda")
    far = 2 ** 31 // D                                   # rows of head 1
    q = big.as_strided((1, 2, N, D), (0, far * D, D, 1))
    q.copy_(randn(g, 1, 2, N, D))
    k = randn(g, 1, 1, N, D).to(torch.bfloat16)
    dq, dk = randn(g, 1, 2, N, D).to(torch.bfloat16), randn(g, 1, 1, N, D).to(torch.bfloat16)
    want = bd.sage_qk_norm_rope_fwd(q.contiguous(), k, w, w, inv)
    got = bd.sage_qk_norm_rope_fwd(q, k, w, w, inv)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want = bd.sage_qk_norm_rope_bwd(q.contiguous(), k, w, w, inv, dq, dk)
    got = bd.sage_qk_norm_rope_bwd(q, k, w, w, inv, dq, dk)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    bd.sage_qk_norm_rope_bwd(q, k, w, w, inv, dq, dk, out=(q, k.clone(), None, None))
    assert torch.equal(q, want[0])
    # many tokens: more rows than 2^31 elements hold
    B, N = 9, 1 << 21
    x = torch.empty((B, 1, N, D), dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        x[b] = randn(g, 1, N, D)
    lens = torch.tensor([N, 0, N, 5, N, N, 1, N, N - 1], dtype=torch.int32, device="cuda")
    z, zk = bd.sage_qk_norm_rope_fwd(x, x[:, :, :], w, w, inv, lens=lens)
    for b in (0, 1, 3, 8):
        part = bd.sage_qk_norm_rope_fwd(x[b:b + 1, :, -64:], x[b:b + 1, :, -64:], w, w, inv, pos=torch.tensor([N - 64], dtype=torch.int32, device="cuda"))
        n = max(0, min(64, int(lens[b]) - (N - 64)))
        assert torch.equal(z[b, 0, -64:][:n], part[0][0, 0, :n]) and bool((zk[b, 0, -64:][n:] == 0).all())


def test_norm_rope_backward_of_two_streams_at_once():
    """Two backwards at a time, each with its own workspace, as one after the other."""
    import torch
    g = gen(21)
    data = []
    for _ in range(2):
        q, k, dq, dk = (randn(g, 1, h, 700, 128).to(torch.bfloat16) for h in (8, 2, 8, 2))
        data.append((q, k, 1 + 0.1 * randn(g, 128), 1 + 0.1 * randn(g, 128), torch.rand(64, generator=g, device="cuda"), dq, dk))
    want = [bd.sage_qk_norm_rope_bwd(*d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = [[] for _ in data]
    for i in range(5):
        for s, d, out in zip(streams, data, got):
            with torch.cuda.stream(s):
                out.append(bd.sage_qk_norm_rope_bwd(*d))
    torch.cuda.synchronize()
    for w, out in zip(want, got):
        assert all(torch.equal(a, b) for o in out for a, b in zip(o, w))
