"""Norms with rotation, the MXFP4 cache and page tables: every refusal happens on the host before any HIP
call, in the C ABI and in the binding; the tests' own definitions against others (no GPU)."""
import os

import numpy as np
import pytest

from paper_2505_11594_amd import binding as bd

import _more_lm as mo

FAKE = 0x10000  # aligned, non-null; never dereferenced because validation fails first
INVALID, WORKSPACE = bd.SAGE_ERR_INVALID_ARG, bd.SAGE_ERR_WORKSPACE
FP4 = bd.SAGE_KV_FP4


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(bd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return bd.lib()


def st(b=4 * 16 * 128, h=16 * 128, n=128):
    return bd._strides(b, h, n)


def rope(L, **kw):
    a = dict(q=FAKE, k=FAKE, qw=FAKE, kw=FAKE, inv=FAKE, rotary=128, pos=None, each=0, lens=None, zq=FAKE, zk=FAKE, B=2, Hq=4,
             Hkv=2, N=16, D=128, eps=1e-6, flags=4, qs=None, ks=None, zqs=None, zks=None)
    a.update(kw)
    return L.sage_qk_norm_rope_fwd(*a.values(), None)


def rope_bwd(L, ws=FAKE, size=1 << 30, **kw):
    a = dict(q=FAKE, k=FAKE, qw=FAKE, kw=FAKE, inv=FAKE, rotary=128, pos=None, each=0, lens=None, gq=FAKE, gk=FAKE, zq=FAKE, zk=FAKE,
             dqw=FAKE, dkw=FAKE, B=2, Hq=4, Hkv=2, N=16, D=128, eps=1e-6, flags=4, qs=None, ks=None, gqs=None, gks=None, zqs=None,
             zks=None)
    a.update(kw)
    return L.sage_qk_norm_rope_bwd(*a.values(), ws, size, None)


ROPES = [dict(q=None), dict(k=FAKE + 8), dict(qw=FAKE + 2), dict(kw=FAKE + 1), dict(inv=None), dict(inv=FAKE + 2), dict(rotary=-8),
         dict(rotary=136), dict(rotary=20), dict(rotary=1), dict(pos=FAKE + 2), dict(each=2), dict(each=-1), dict(lens=FAKE + 2), dict(zq=None), dict(zk=FAKE + 8),
         dict(B=0), dict(Hq=3), dict(Hkv=0), dict(Hq=1 << 17, Hkv=1 << 17), dict(N=0), dict(D=96), dict(D=256), dict(B=1 << 15, N=1 << 16), dict(eps=0.0),
         dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-35), dict(flags=8), dict(flags=FP4), dict(qs=st(n=132)),
         dict(ks=st(h=-8)), dict(zqs=st(n=64)), dict(zks=st(h=0)), dict(zqs=st(b=0)), dict(zks=st(b=1 << 41))]


@pytest.mark.parametrize("bad", ROPES)
def test_norm_rope_refusals(L, bad):
    assert rope(L, **bad) == INVALID
    assert rope_bwd(L, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(gq=None), dict(gk=FAKE + 4), dict(dqw=FAKE + 2), dict(dkw=FAKE + 1), dict(gqs=st(n=7)), dict(ws=None),
                                 dict(ws=FAKE + 16)])
def test_norm_rope_backward_refusals(L, bad):
    assert rope_bwd(L, **bad) == INVALID


def test_norm_rope_backward_workspace(L):
    need = bd.qk_norm_rope_bwd_workspace_size(2, 4, 2, 16, 128)
    assert 0 < need <= 1 << 20 and need % 256 == 0
    assert bd.qk_norm_rope_bwd_workspace_size(1, 64, 8, 1 << 20, 128) <= 1 << 20
    assert rope_bwd(L, size=need - 1) == WORKSPACE
    for bad in ((0, 4, 2, 16, 128), (2, 4, 3, 16, 128), (2, 4, 2, 0, 128), (2, 4, 2, 16, 80), (1 << 15, 4, 2, 1 << 16, 64)):
        assert bd.qk_norm_rope_bwd_workspace_size(*bad) == 0


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, ks=(2 * 16 * 64, 16 * 64, 64), vs=(2 * 16 * 64, 16 * 64, 64), pages=10, page_size=16,
             Hkv=2, D=128)
    a.update(kw)
    return bd._cache(*[x for v in a.values() for x in (v if isinstance(v, tuple) else (v,))])


def append(L, c=None, **kw):
    a = dict(k=FAKE, v=FAKE, ks=None, vs=None, table=FAKE, M=4, pos=FAKE, counts=None, weights=None, ws=0, S=2, N=3, flags=4 | FP4)
    a.update(kw)
    return L.sage_kv_append(c or cache(), *a.values(), None)


def append_slots(L, c=None, **kw):
    a = dict(k=FAKE, v=FAKE, ks=None, vs=None, slots=FAKE, B=2, N=3, flags=4 | FP4)
    a.update(kw)
    return L.sage_kv_append_slots(c or cache(), *a.values(), None)


def decode(L, c=None, **kw):
    a = dict(q=FAKE, qss=4 * 128, qsh=128, o=FAKE, lse=None, table=FAKE, M=4, lens=FAKE, S=2, Hq=4, window=64, sinks=0, weights=None,
             wstride=0, flags=4 | FP4, ws=FAKE, size=1 << 30)
    a.update(kw)
    return L.sage_attn_paged_decode(c or cache(), *a.values(), None)


@pytest.mark.parametrize("bad", [dict(k=0), dict(v=FAKE + 8), dict(k_scale=0), dict(k_scale=0, v_scale=0), dict(v_scale=FAKE + 2), dict(pages=0),
                                 dict(page_size=0), dict(page_size=(1 << 30) + 1), dict(Hkv=0), dict(D=96), dict(ks=(2048, 1024, 72)), dict(vs=(-16, 1024, 64))])
def test_fp4_cache_refusals(L, bad):
    for f in (append, append_slots, decode):
        assert f(L, cache(**bad)) == INVALID, f.__name__


@pytest.mark.parametrize("bad", [dict(ks=(2048, 1024, 48)), dict(vs=(0, 1024, 64)), dict(vs=(2048, 0, 64))])
def test_written_fp4_caches_have_no_rows_in_common(L, bad):
    for f in (append, append_slots):
        assert f(L, cache(**bad)) == INVALID, f.__name__


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=FAKE + 8), dict(slots=None), dict(slots=FAKE + 4), dict(B=0), dict(B=65536), dict(N=0),
                                 dict(N=1 << 30), dict(flags=8), dict(flags=FP4 | 0x400), dict(ks=st(n=12)), dict(vs=st(b=-8))])
def test_append_slots_refusals(L, bad):
    assert append_slots(L, **bad) == INVALID
    assert append_slots(L, cache(), flags=4, B=0) == INVALID


def evict(L, c=None, f="sage_kv_evict_fp4", **kw):
    a = dict(table=FAKE, M=4, lens=FAKE, weights=FAKE, wstride=64, new_table=FAKE, M2=2, budget=20, first=2, last=3, new_lens=FAKE + 4096,
             new_weights=FAKE + 4096, kept=FAKE, S=2, ws=FAKE, size=1 << 30)
    a.update(kw)
    return getattr(L, f)(c or cache(), *a.values(), None)


def test_decode_over_fp4_refusals(L):
    wide = cache(page_size=64, ks=(8192, 4096, 64), vs=(8192, 4096, 64))
    assert decode(L, weights=FAKE, wstride=63) == INVALID
    assert decode(L, weights=FAKE + 2, wstride=64) == INVALID
    assert decode(L, weights=FAKE, wstride=64, ws=None) == INVALID
    assert decode(L, flags=FP4 | 8) == INVALID
    # the workspace is the one that the size function gives for any cache
    for w in (False, True):
        need = bd.attn_paged_decode_workspace_size(3, 16, 2, 128, 100, 64, w)
        kw = dict(weights=FAKE, wstride=6400) if w else {}
        assert decode(L, wide, S=3, Hq=16, M=100, size=need - 1, **kw) == WORKSPACE


@pytest.mark.parametrize("bad", [dict(k=0), dict(v=FAKE + 8), dict(k_scale=0), dict(k_scale=0, v_scale=0), dict(v_scale=FAKE + 2), dict(D=96),
                                 dict(ks=(2048, 1024, 72)), dict(vs=(-16, 1024, 64)), dict(ks=(2048, 1024, 48)), dict(vs=(2048, 0, 64))])
def test_evict_refuses_bad_fp4_caches(L, bad):
    assert evict(L, cache(**bad)) == INVALID


@pytest.mark.parametrize("bad", [dict(lens=None), dict(weights=None), dict(weights=FAKE + 2), dict(new_table=None), dict(budget=0), dict(budget=33),
                                 dict(first=18), dict(last=-1), dict(M2=0), dict(wstride=63), dict(new_lens=FAKE), dict(new_weights=FAKE),
                                 dict(kept=FAKE + 1), dict(S=70000), dict(ws=None, M=2000, wstride=32000), dict(ws=FAKE + 64, M=2000, wstride=32000)])
def test_evict_over_fp4_refusals(L, bad):
    assert evict(L, **bad) == INVALID
    # rows of 64 bytes overlap as rows of 128 int8 values do
    assert evict(L, f="sage_kv_evict") == INVALID


def plan(L, **kw):
    a = dict(table=FAKE, M=4, lens=FAKE, counts=FAKE + 4096, free=FAKE, F=10, n_free=FAKE, page=16, granted=FAKE, starts=FAKE, pos=FAKE,
             slots=FAKE, T=10, S=3)
    a.update(kw)
    return L.sage_kv_plan(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(table=None), dict(M=0), dict(lens=FAKE + 2), dict(counts=None), dict(counts=FAKE), dict(free=None),
                                 dict(F=0), dict(n_free=None), dict(page=0), dict(M=1 << 20, page=1 << 20), dict(granted=None), dict(starts=FAKE + 1),
                                 dict(pos=None), dict(slots=None), dict(slots=FAKE + 4), dict(T=0), dict(T=(1 << 30) + 1), dict(S=0), dict(S=65536)])
def test_plan_refusals(L, bad):
    assert plan(L, **bad) == INVALID


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch
    q, k = torch.zeros((1, 4, 8, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16)
    w, inv = torch.ones(64), torch.ones(32)
    with pytest.raises(ValueError):
        bd.sage_qk_norm_rope_fwd(q, k, w, w, inv)
    with pytest.raises(TypeError):
        bd.sage_qk_norm_rope_fwd(q.float(), k.float(), w, w, inv)
    with pytest.raises(ValueError):
        bd.sage_qk_norm_rope_bwd(q, k, w, w, inv, q, k)
    codes, sc = torch.zeros((4, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 16, 2), dtype=torch.uint8)
    table, lens = torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        bd.sage_kv_append_slots(k, k, codes, codes, torch.zeros((1, 8), dtype=torch.int64), k_scale=sc, v_scale=sc)
    with pytest.raises(ValueError):
        bd.sage_attn_paged_decode(q[:, :, 0], codes, codes, table, lens, k_scale=sc, v_scale=sc)
    with pytest.raises(ValueError):
        bd.sage_kv_plan(table, lens, lens.clone(), torch.zeros(4, dtype=torch.int32), lens[:1].clone(), 16, 8)


def test_formulas_against_differentiation_and_complex_numbers():
    import torch
    g = torch.Generator().manual_seed(2)
    x, w, dz = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((2, 3, 5, 64), (64,), (2, 3, 5, 64)))
    p, inv = torch.randint(0, 100, (2, 5), generator=g), torch.rand(12, generator=g)
    live = torch.ones((2, 1, 5, 1), dtype=torch.bool)
    live[1, 0, 3:] = False
    th = mo.angles(inv, p)[:, None]
    x.requires_grad_(True), w.requires_grad_(True)
    for pairs in (False, True):
        y, z = mo.norm_rope(x, w, th, pairs, 1e-5, live)
        a, b = mo.pair(y, 24, pairs)
        turned = torch.complex(a, b) * torch.polar(torch.ones_like(th), th) * live
        za, zb = mo.pair(z, 24, pairs)
        assert torch.allclose(turned.real, za, atol=1e-13) and torch.allclose(turned.imag, zb, atol=1e-13)
        gx, gw = torch.autograd.grad(z, (x, w), dz)
        dx, dw, _, _ = mo.norm_rope_grads(x.detach(), w.detach(), th, pairs, 1e-5, live, dz, p, 2.0 ** -8)
        assert torch.allclose(torch.where(live, dx, 0.0), gx, atol=1e-12) and torch.allclose(dw, gw, atol=1e-11)


def test_fp4_rows_against_the_oracle():
    """Rows in MXFP4 as the attention's own quantizer defines them."""
    import torch
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 64)) * 2.0 ** rng.integers(-30, 30, (40, 2)).repeat(32, 1)
    x[0, :32] = 0
    x[1] = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 8)
    x = torch.from_numpy(x).bfloat16().double().numpy()
    codes, scale = mo.fp4_rows(x)
    e = scale.astype(int) - 127
    top = np.abs(x).reshape(40, 2, 32).max(-1)
    assert (6 * 2.0 ** e >= top).all() and ((6 * 2.0 ** (e - 1.0) < top) | (e == -127)).all()
    v = mo.fp4_values(torch.from_numpy(codes), torch.from_numpy(scale)).numpy()
    grid = np.array(mo.VALUES + [-y for y in mo.VALUES])
    best = np.abs(x[..., None] / 2.0 ** e.repeat(32, -1)[..., None].astype(float) - grid).min(-1)
    assert (np.abs(x - v) / 2.0 ** e.repeat(32, -1).astype(float) == best).all()


def test_plan_against_the_rules():
    """No page twice, none lost; positions and slots of what was granted; nobody passed over for pages."""
    rng = np.random.default_rng(1)
    for _ in range(50):
        S, M, page, F = 9, 5, 4, 60
        had = rng.integers(0, 12, S).astype(np.int32)
        held = -(-had // page)
        ids = rng.permutation(F).astype(np.int32)
        table, i = np.full((S, M), -1, np.int32), 0
        for s in range(S):
            table[s, :held[s]], i = ids[i:i + held[s]], i + int(held[s])
        free = np.concatenate([ids[i:], np.zeros(i, np.int32)])
        n = int(rng.integers(0, F - i + 1))
        counts = rng.integers(-2, 9, S).astype(np.int32)
        t2, l2, f2, n2, granted, starts, pos, slots = mo.plan(table, had, counts, free, [n], page, 30)
        pool = sorted(list(free[:n]) + list(table[table >= 0]))
        assert sorted(list(f2[:n2[0]]) + list(t2[t2 >= 0])) == pool
        assert (l2 == np.where(counts < 0, 0, had + granted)).all() and starts[-1] == granted.sum() <= 30
        assert ((t2 >= 0).sum(1) == -(-l2 // page)).all()
        refused = [s for s in range(S) if counts[s] > 0 and granted[s] == 0 and had[s] + counts[s] <= M * page]
        if refused:
            later = [s for s in range(refused[0], S) if granted[s] > 0]
            assert all(-(-int(l2[s]) // page) == held[s] for s in later)
        live = slots[:starts[-1]]
        assert len(set(live.tolist())) == len(live) and (live >= 0).all() and (slots[starts[-1]:] == -1).all()
