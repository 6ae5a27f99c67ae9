"""Steps of a batch of requests that come, wait, are refused, bring several tokens and end: page tables, norms with
rotation, storing by slots and the attention of every request's last token, captured, replayed, and checked at every step
against the attention over each request's own tokens, kept apart from any cache."""
import numpy as np
import pytest

from paper_2505_11594_amd import binding as bd

import _lm
import _more_lm as mo
from _gpu import torch_dev, say

pytestmark = pytest.mark.gpu


def step_of(st):
    """One step.  The plan packs the granted tokens of all requests; the attention takes a row per request, that of its
    last token: starts[s + 1] - 1.  (A request that was granted none has no new token, and its row says nothing.)"""
    granted, starts, pos, slots = bd.sage_kv_plan(st["table"], st["lens"], st["counts"], st["free"], st["n_free"], st["page"], st["T"])
    zq, zk = bd.sage_qk_norm_rope_fwd(st["q"], st["k"], st["wq"], st["wk"], st["inv"], pos=pos[None])
    sc = dict(k_scale=st["k_scale"], v_scale=st["v_scale"])
    bd.sage_kv_append_slots(zk, st["v"], st["k_cache"], st["v_cache"], slots[None], **sc)
    last = (starts[1:] - 1).clamp(min=0).long()
    o, lse = bd.sage_attn_paged_decode(zq[0].transpose(0, 1)[last], st["k_cache"], st["v_cache"], st["table"], st["lens"], **sc)
    return granted, starts, pos, slots, zq, zk, o, lse


def stored(x, kind):
    """What a cache holds of rows [Hkv, D] of new tokens, in 64 bits."""
    import torch
    if kind == "16":
        return x.double()
    if kind == "int8":
        codes, s = _lm.quantized(x)
        return codes.double() * s.double()[..., None]
    codes, scale = mo.fp4_rows(x.double().cpu().numpy())
    return mo.fp4_values(torch.from_numpy(codes), torch.from_numpy(scale)).to(x.device)


def bounds(q, kr, vr, kind, u):
    import torch
    has, D, n = torch.ones(len(kr), dtype=torch.bool, device=q.device), q.shape[-1], len(kr)
    if kind == "fp4":
        r = mo.fp4_decode(q, kr, vr, has, None, 0)
        return r, _lm.o_bound(r, n, u, 2.0 ** -16), _lm.lse_bound(r, n)
    r = _lm.decode_attention(q, kr, vr, has, None, 0)
    r["e"] = r["e"] * 1.1 + 2.0 ** -22 * r["e"] / 2.0 ** -24 / (D + 4)   # the scale's product
    return r, _lm.o_bound(r, n, u, (_lm.unit(torch.bfloat16) if kind == "int8" else u) ** 2), _lm.lse_bound(r, n)


@pytest.mark.parametrize("kind,dtype,D", [("16", "bfloat16", 64), ("16", "float16", 128), ("int8", "bfloat16", 128), ("int8", "float16", 64),
                                          ("fp4", "bfloat16", 64), ("fp4", "float16", 128)])
def test_steps_of_requests_that_come_wait_and_end(kind, dtype, D):
    torch = torch_dev()
    g = torch.Generator(device="cuda").manual_seed(78)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    S, Hq, Hkv, page, M, P, T = 6, 8, 2, 16, 8, 11, 11
    dt = getattr(torch, dtype)

    def state():
        x = torch.Generator(device="cuda").manual_seed(5)
        i32 = dict(dtype=torch.int32, device="cuda")
        shape = (P, Hkv, page, D // 2 if kind == "fp4" else D)
        ct = {"16": dt, "int8": torch.int8, "fp4": torch.uint8}[kind]
        st = dict(k_cache=torch.zeros(shape, dtype=ct, device="cuda"), v_cache=torch.zeros(shape, dtype=ct, device="cuda"), k_scale=None,
                  v_scale=None, page=page, T=T, table=torch.full((S, M), -1, **i32), lens=torch.zeros(S, **i32), counts=torch.ones(S, **i32),
                  free=torch.randperm(P, generator=x, device="cuda").to(torch.int32), n_free=torch.full((1,), P, **i32),
                  q=torch.zeros((1, Hq, T, D), dtype=dt, device="cuda"), k=torch.zeros((1, Hkv, T, D), dtype=dt, device="cuda"),
                  v=torch.zeros((1, Hkv, T, D), dtype=dt, device="cuda"), wq=torch.rand(D, generator=x, device="cuda") + 0.5,
                  wk=torch.rand(D, generator=x, device="cuda") + 0.5, inv=(10000.0 ** (-torch.arange(0, D, 2, device="cuda").double() / D)).float())
        if kind != "16":
            s, sd = ((P, Hkv, page), torch.float32) if kind == "int8" else ((P, Hkv, page, D // 32), torch.uint8)
            st.update(k_scale=torch.zeros(s, dtype=sd, device="cuda"), v_scale=torch.zeros(s, dtype=sd, device="cuda"))
        return st

    eager, replayed = state(), state()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step_of(state())                                 # (warms the library up, on another state)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step_of(replayed)

    rng, u = np.random.default_rng(6), _lm.unit(dt)
    history = [[] for _ in range(S)]                     # per request: what a cache holds of each token's k and v
    seen, worst = dict(ended=0, waited=0, refused=0, no_pages=0, several=0, moved=0), [0.0, 0.0]
    for it in range(60):
        counts = rng.choice([1] * 8 + [0, 4, 4, -1], S).tolist()
        counts = [(0 if not h else -1 if rng.random() < 0.5 else 1) if c < 0 else c for c, h in zip(counts, history)]
        q, k, v = (rn(*eager[x].shape).to(dt) for x in "qkv")
        for st in (eager, replayed):
            st["q"].copy_(q), st["k"].copy_(k), st["v"].copy_(v)
            st["counts"].copy_(torch.tensor(counts, dtype=torch.int32))
        before = [eager[x].cpu().numpy() for x in ("table", "lens", "counts", "free", "n_free")]
        want = step_of(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), it
        for x in ("table", "lens", "free", "n_free", "k_cache", "v_cache", "k_scale", "v_scale"):
            assert eager[x] is None or torch.equal(eager[x], replayed[x]), (it, x)
        granted, starts, pos, slots, _, zk, o, lse = want
        zq = want[4]
        ref = mo.plan(*before, page, T)
        for a, b in zip((eager["table"], eager["lens"], eager["free"], eager["n_free"], granted, starts, pos, slots), ref):
            assert (a.cpu().numpy() == b).all(), it
        granted, starts = granted.tolist(), starts.tolist()
        for s, c in enumerate(counts):
            seen["ended"] += c < 0
            seen["waited"] += c == 0 and bool(history[s])
            seen["refused"] += c > 0 and granted[s] == 0
            seen["no_pages"] += c > 0 and granted[s] == 0 and sum(x for x in counts if x > 0) <= T
            seen["several"] += granted[s] > 1
            seen["moved"] += granted[s] > 0 and starts[s + 1] - 1 != s
            if c < 0:
                history[s] = []
            for i in range(granted[s]):
                row = starts[s] + i
                assert int(pos[row]) == len(history[s])
                history[s].append((stored(zk[0, :, row], kind), stored(v[0, :, row], kind)))
        assert eager["lens"].tolist() == [len(h) for h in history]
        for s in range(S):
            if granted[s] == 0:
                continue
            for h in range(Hkv):
                kr, vr = (torch.stack([t[j][h] for t in history[s]]) for j in range(2))
                hs = slice(h * Hq // Hkv, (h + 1) * Hq // Hkv)
                r, to, tl = bounds(zq[0, hs, starts[s + 1] - 1].double(), kr, vr, kind, u)
                worst[0] = max(worst[0], float(((o[s, hs].double() - r["o"]).abs() / to).max()))
                worst[1] = max(worst[1], float(((lse[s, hs].double() - r["lse"]).abs() / tl).max()))
        assert max(worst) <= 1, (it, worst)
    say("%s %s D %d: O at %.3f of its bound, L at %.3f; %s" % (kind, dtype, D, *worst, seen))
    assert min(seen.values()) >= 5
