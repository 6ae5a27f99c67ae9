"""GPU checks of the language-model operators where their inputs or sizes are at an edge:
infinities and NaN that a row does see, and calls far larger than those of test_gpu_lm.py."""
import math

import pytest

from paper_2505_11594_amd import binding as bd

import _lm
import _slopes
from _gpu import say
from test_gpu_lm import DT, WINDOWS, check_grads, gen, make_cache, qkv, randn

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


# ---------------------------------------------------------------- values that are seen and not finite
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,page,lens", [(64, 16, [40, 7]), (128, 24, [300, 129]), (128, 64, [3000, 700]), (64, 16, [9000, 1])])
def test_paged_decode_infinities_and_nan_that_are_seen(D, page, lens, dtype):
    """A value that is no finite number, seen by every head of its key head: its channel is that
    infinity, or NaN where there are both or a NaN; every other output keeps the bits that it has
    with 0 in the value's place."""
    import torch
    g = gen(7 * D + lens[0])
    Hq, Hkv, ch = 8, 2, D // 2 + 3
    c, table, _ = make_cache(g, len(lens), Hkv, page, D, lens, dtype, False)
    q = randn(g, len(lens), Hq, D).to(getattr(torch, DT[dtype]))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    v = c["v_cache"]
    run = lambda: bd.sage_attn_paged_decode(q, c["k_cache"], v, table, ln)
    n = lens[0]
    for puts, want in (([(0, INF)], INF), ([(n - 1, -INF)], -INF), ([(n // 2, NAN)], NAN), ([(3, INF), (n // 2, -INF)], NAN),
                       ([(n // 3, INF), (n // 2, INF)], INF), ([(n // 3, -INF), (n - 1, NAN)], NAN)):
        where = [(int(table[0, j // page]), 1, j % page, ch) for j, _ in puts]
        old = [v[w].clone() for w in where]
        for w in where:
            v[w] = 0
        o0, l0 = run()
        for w, (_, x) in zip(where, puts):
            v[w] = x
        o, l = run()
        torch.cuda.synchronize()
        say("seen %s: %s" % (puts, o[0, :, ch].tolist()))
        got = o[0, Hq // 2:, ch].float()
        assert torch.equal(got.nan_to_num(7, 8, 9), torch.full_like(got, want).nan_to_num(7, 8, 9))
        o[0, Hq // 2:, ch] = o0[0, Hq // 2:, ch]
        assert torch.equal(o, o0) and torch.equal(l, l0)
        for w, x in zip(where, old):
            v[w] = x


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [200, 3000])
def test_paged_decode_infinity_of_a_token_with_hardly_any_weight(n, dtype):
    """The first half of the sequence has scores 512 below the other's: weights that are 0 in fp32, and
    whole parts of the split whose factor is.  An infinity there is seen all the same."""
    import torch
    g = gen(n)
    D, page = 64, 16
    c, table, _ = make_cache(g, 1, 1, page, D, [n], dtype, False)
    k, v = c["k_cache"], c["v_cache"]
    ids = table[0].long()
    half = -(-n // (2 * page))
    k[ids[:half]], k[ids[half:]] = -8.0, 0.0             # scores -64 * 8 * 8 / 8 and 0
    q = torch.full((1, 4, D), 8.0, dtype=k.dtype, device="cuda")
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    o0, l0 = bd.sage_attn_paged_decode(q, k, v, table, ln)
    for at, bad in ((5, INF), (page * (half - 1) + 1, -INF), (40, NAN)):
        v2 = v.clone()
        v2[int(ids[at // page]), 0, at % page, 9] = bad
        o, l = bd.sage_attn_paged_decode(q, k, v2, table, ln)
        torch.cuda.synchronize()
        got = o[0, :, 9].float()
        assert torch.equal(got.nan_to_num(7, 8, 9), torch.full_like(got, bad).nan_to_num(7, 8, 9)), (at, bad, got.tolist())
        o[0, :, 9] = o0[0, :, 9]
        assert torch.equal(o, o0) and torch.equal(l, l0)


# ---------------------------------------------------------------- the power of two of fp16's dS
@pytest.mark.parametrize("at", [(0, 0), (7, 640), (15, 1099)])
@pytest.mark.parametrize("what", ["dout", "v"])
def test_window_backward_fp16_scale_knows_every_row(what, at):
    """One row of dO or V is 2^9 times the others, in any block of any head of the group: dS of that
    size would pass fp16's range if the bound had missed it."""
    import torch
    q, k, v = qkv(5, 1, 16, 1, 1100, 64, "fp16")
    dout = randn(gen(6), 1, 16, 1100, 64).half()
    (dout if what == "dout" else v)[0, at[0] if what == "dout" else 0, at[1]] *= 512
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=200, sinks=3)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=200, sinks=3)
    torch.cuda.synchronize()
    check_grads(q, k, v, dout, grads, 200, 3, None, "%s large at %s" % (what, at))


def test_window_backward_fp16_takes_no_longer_than_bf16_as_lengths_grow():
    """16 query heads of one key head under a short window: the work per workgroup is the same at any
    length.  (fp16 took 2.2 times bf16's time here when every wave looked for the scale itself.)"""
    import torch
    N = 32768
    times = []
    for dt in (torch.float16, torch.bfloat16):
        q, k, v, dout = (torch.randn((1, h, N, 64), device="cuda").to(dt) for h in (16, 1, 1, 16))
        o, lse = bd.sage_attn_window_fwd(q, k, v, window=64)
        ws = torch.empty(bd.attn_window_bwd_workspace_size(1, 16, 1, N, 64, 64), dtype=torch.uint8, device="cuda")
        out = [torch.empty_like(x) for x in (q, k, v)]
        best = math.inf
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=64, workspace=ws, out=out)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) / 5 * 1e3)
        times.append(best)
    say("backward of 32768 tokens, window 64: fp16 %.0f us, bf16 %.0f us" % tuple(times))
    assert times[0] < 1.5 * times[1]


# ---------------------------------------------------------------- gradients against slopes
@pytest.mark.parametrize("case", [c for c in WINDOWS if c[3] > 1])
def test_window_gradients_are_slopes_of_the_definition(case):
    """Each gradient against the slope of the definition along it (_slopes.py).  A gradient of zero is
    off by the slope itself, so it would not pass where the tolerance is less than that."""
    import torch
    B, Hq, Hkv, N, D, dtype, window, sinks, lens = case
    q, k, v = qkv(13 + N + D, B, Hq, Hkv, N, D, dtype)
    dout = randn(gen(N + 1), B, Hq, N, D).to(q.dtype)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=window, sinks=sinks, lens=ln)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=window, sinks=sinks, lens=ln)
    torch.cuda.synchronize()
    want, bound = check_grads(q, k, v, dout, grads, window, sinks, lens, "slopes %s" % (case,))
    u = _lm.unit(q.dtype)
    bound = [t + u * (w.abs() + t) + torch.finfo(q.dtype).smallest_normal * 2.0 ** -10 for w, t in zip(want, bound)]
    ratios, sizes = _slopes.slopes_agree([x.double() for x in (q, k, v)], dout.double(), grads, want, bound, window, sinks, lens)
    say("slopes: %s of the tolerances, which are %s of the slopes" % (ratios, sizes))
    first = 2 if window == 1 and sinks == 0 else 0       # (a query that sees one key: dQ and dK are 0)
    assert max(ratios) <= 1 and max(sizes[first:]) < 1


# ---------------------------------------------------------------- large calls
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_window_tensors_of_more_than_2_31_elements(dtype):
    """262181 tokens of 72 heads: the last group's last rows and keys against the definition over the
    sinks and the last tokens, of which the first see less than they should and are left out."""
    import torch
    Hq, Hkv, N, D, window, sinks = 72, 8, 2 ** 18 + 37, 128, 100, 4
    G, dt = Hq // Hkv, getattr(torch, DT[dtype])
    assert Hq * N * D > 2 ** 31
    g = gen(91)
    rnd = lambda h: torch.randn((1, h, N, D), generator=g, device="cuda", dtype=dt)
    q, k, v, dout = rnd(Hq), rnd(Hkv), rnd(Hkv), rnd(Hq)
    say("window %d tokens %s" % (N, dtype))
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=window, sinks=sinks)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=window, sinks=sinks)
    torch.cuda.synchronize()
    first = N - sinks - (N - sinks) % 128 - 512          # tiles lie in the short sequence as in the long one
    at = torch.cat([torch.arange(sinks), torch.arange(first + sinks, N)]).cuda()
    n, whole, u = len(at), slice(sinks + window, None), _lm.unit(dt)
    short = lambda x, h: x[0, h, at].double()
    kk, vv = short(k, -1), short(v, -1)
    sums = {x: torch.zeros_like(kk) for x in ("dk", "dv", "edk", "edv")}
    worst = [0.0] * 5
    over = lambda got, w, t: float(((got.double() - w).abs() / t)[whole].max())
    for h in range(Hq - G, Hq):
        r = _lm.window_attention(short(q, h), kk, vv, window, sinks, n, short(dout, h), u)
        worst[0] = max(worst[0], over(o[0, h, at], r["o"], _lm.o_bound(r, n, u)))
        worst[1] = max(worst[1], over(lse[0, h, at], r["lse"], _lm.lse_bound(r, n)))
        t = r["edq"] + u * (r["dq"].abs() + r["edq"]) + 1e-9
        worst[2] = max(worst[2], over(grads[0][0, h, at], r["dq"], t))
        for x in sums:
            sums[x] += r[x]
    for i, x in ((3, "dk"), (4, "dv")):
        t = sums["e" + x] + u * (sums[x].abs() + sums["e" + x]) + 1e-9
        worst[i] = over(grads[i - 2][0, -1, at], sums[x], t)
    say("O, L, dQ, dK, dV at %s of their bounds" % worst)
    assert max(worst) <= 1


def test_window_strides_of_more_than_2_31_elements():
    """Rows 2^22 elements apart, the largest token stride that is taken: the bits of contiguous copies."""
    import torch
    B, Hq, Hkv, N, D = 2, 4, 2, 700, 128
    q, k, v = qkv(92, B, Hq, Hkv, N, D, "bf16")
    dout = randn(gen(93), B, Hq, N, D).to(q.dtype)
    o, lse = bd.sage_attn_window_fwd(q, k, v, window=90, sinks=40)
    grads = bd.sage_attn_window_bwd(q, k, v, o, lse, dout, window=90, sinks=40)
    big = torch.empty((N, B, 2 ** 21 // 1024, 1024), dtype=q.dtype, device="cuda")
    assert big.numel() > 2 ** 31
    far = []
    for i, x in enumerate((q, k, v, o, dout)):
        y = big[:, :, -1 - i, :x.shape[1] * D].unflatten(-1, (x.shape[1], D)).permute(1, 2, 0, 3)
        assert y.shape == x.shape and y.stride(2) == 2 ** 22
        if x is not o:
            y.copy_(x)
        far.append(y)
    say("window, rows 2^22 elements apart")
    o2, lse2 = bd.sage_attn_window_fwd(*far[:3], window=90, sinks=40, out=far[3])
    got = bd.sage_attn_window_bwd(*far[:4], lse2, far[4], window=90, sinks=40)
    torch.cuda.synchronize()
    assert torch.equal(o2, o) and torch.equal(lse2, lse) and all(torch.equal(a, b) for a, b in zip(got, grads))
