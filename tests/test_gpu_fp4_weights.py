"""Attention weights over an MXFP4 cache for more sequences than a wave has lanes: the steps before each sequence come
from a launch of their own then, and the workspace holds them beside the sums and the kept scores."""
import numpy as np
import pytest

from paper_2505_11594_amd import binding as bd

from _gpu import say
from test_gpu_more_lm import check_decode, fp4_cache, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,Hq,Hkv,D,page,dtype,window,sinks", [
    (64, 8, 2, 64, 16, "bfloat16", None, 0), (65, 8, 2, 64, 16, "bfloat16", None, 0), (65, 8, 1, 128, 24, "float16", 300, 5),
    (130, 16, 1, 128, 32, "float16", 700, 70), (300, 4, 1, 64, 16, "bfloat16", 400, 3), (300, 20, 1, 64, 16, "float16", None, 0)])
def test_weights_of_many_ragged_sequences(S, Hq, Hkv, D, page, dtype, window, sinks):
    import torch
    g = gen(S + D + page)
    lens = [int(x) for x in np.random.default_rng(S).integers(0, 1500, S)]
    lens[0], lens[1], lens[2], lens[62], lens[-1] = 0, 0, 1, 1499, 0
    lens[S // 2] = 0
    c, table, _ = fp4_cache(g, S, Hkv, page, D, lens)
    q = (0.5 * randn(g, S, Hq, D)).to(getattr(torch, dtype))
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table[3, 0] = -1                                     # a hole
    M = table.shape[1]
    w0 = torch.rand((S, Hkv, M * page + 3), generator=g, device="cuda")
    kw = dict(window=window, sinks=sinks, k_scale=c["k_scale"], v_scale=c["v_scale"])
    args = (q, c["k_cache"], c["v_cache"], table, ln)
    say("weights of %d sequences" % S)
    got = []
    for fill in (0xFF, 0):                               # whatever the workspace held before
        ws = torch.full((bd.attn_paged_decode_workspace_size(S, Hq, Hkv, D, M, page, True),), fill, dtype=torch.uint8, device="cuda")
        w1 = w0.clone()
        got.append(tuple(bd.sage_attn_paged_decode(*args, weights=w1, workspace=ws, **kw)) + (w1,))
    plain = bd.sage_attn_paged_decode(*args, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    o, lse, w1 = got[0]
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
    # nothing is added where nothing is seen
    j = torch.arange(w0.shape[2], device="cuda")
    see = j < ln[:, None]
    if window is not None:
        see = see & ((j >= ln[:, None] - window) | (j < sinks))
    assert torch.equal(torch.where(see[:, None], w0, w1), w0)
    pick = sorted({i % S for i in (0, 1, 2, 3, 31, 62, 63, 64, S // 2, S // 2 + 1, -3, -2, -1)})
    at = torch.tensor(pick, device="cuda")
    check_decode(q[at], c, table[at], [lens[i] for i in pick], window, sinks, o[at], lse[at], "%d sequences" % S, w0[at], w1[at])
