"""Window attention, paged cache, one-token attention and eviction: every refusal
happens on the host before any HIP call, in the C ABI and in the binding (no GPU)."""
import os

import pytest

from paper_2505_11594_amd import binding as bd

FAKE = 0x10000  # aligned, non-null; never dereferenced because validation fails first
INVALID, WORKSPACE = bd.SAGE_ERR_INVALID_ARG, bd.SAGE_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(bd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return bd.lib()


def st(b=4 * 128 * 128, h=128 * 128, n=128):
    return bd._strides(b, h, n)


def fwd(L, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=None, lens=None, B=1, Hq=4, Hkv=2, N=128, D=128, window=64, sinks=0, flags=4,
             qs=None, ks=None, vs=None, os=None)
    a.update(kw)
    return L.sage_attn_window_fwd(*a.values(), None)


def bwd(L, ws=FAKE, size=1 << 40, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dout=FAKE, lens=None, dq=FAKE, dk=FAKE, dv=FAKE, B=1, Hq=4, Hkv=2,
             N=128, D=128, window=64, sinks=0, flags=4, qs=None, ks=None, vs=None, os=None, gs=None)
    a.update(kw)
    return L.sage_attn_window_bwd(*a.values(), ws, size, None)


SHAPES = [dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(N=0), dict(D=96), dict(D=256), dict(window=0), dict(window=-1),
          dict(sinks=-1), dict(flags=8), dict(flags=0x10), dict(N=(1 << 24) + 1), dict(Hq=1 << 17, Hkv=1 << 17), dict(q=None),
          dict(v=None), dict(k=FAKE + 8), dict(lens=FAKE + 2), dict(qs=st(n=132)), dict(ks=st(n=-128)), dict(vs=st(n=(1 << 22) + 8)),
          dict(qs=st(b=1 << 41))]


@pytest.mark.parametrize("bad", SHAPES + [dict(o=None), dict(o=FAKE + 4), dict(lse=FAKE + 1), dict(os=st(n=64)), dict(os=st(h=0)),
                                          dict(os=st(h=127 * 128))])
def test_window_forward_refusals(L, bad):
    assert fwd(L, **bad) == INVALID


@pytest.mark.parametrize("bad", SHAPES + [dict(o=None), dict(lse=None), dict(dout=None), dict(dq=FAKE + 8), dict(dk=None),
                                          dict(dv=FAKE + 2), dict(gs=st(n=7)), dict(ws=None), dict(ws=FAKE + 16),
                                          dict(B=9000, Hq=8, Hkv=1, N=1)])
def test_window_backward_refusals(L, bad):
    assert bwd(L, **bad) == INVALID


def test_window_backward_workspace(L):
    need = bd.attn_window_bwd_workspace_size(2, 8, 2, 1000, 64, 100, 5)
    assert need > 2 * 2 * 8 * 1000 * 4
    assert bwd(L, size=need - 1, B=2, Hq=8, Hkv=2, N=1000, D=64, window=100, sinks=5) == WORKSPACE
    # a window over everything leaves no sinks to keep parts of
    assert bd.attn_window_bwd_workspace_size(2, 8, 2, 1000, 64, None, 5) == bd.attn_window_bwd_workspace_size(2, 8, 2, 1000, 64)
    for bad in ((0, 8, 2, 10, 64), (1, 8, 3, 10, 64), (1, 8, 2, 10, 80)):
        assert bd.attn_window_bwd_workspace_size(*bad) == 0


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=0, v_scale=0, ks=(2 * 16 * 128, 16 * 128, 128), vs=(2 * 16 * 128, 16 * 128, 128),
             pages=10, page_size=16, Hkv=2, D=128)
    a.update(kw)
    a = [x for v in a.values() for x in (v if isinstance(v, tuple) else (v,))]
    return bd._cache(*a)


def append(L, c=None, **kw):
    a = dict(k=FAKE, v=FAKE, ks=None, vs=None, table=FAKE, M=4, pos=FAKE, counts=None, weights=None, ws=0, S=2, N=3, flags=4)
    a.update(kw)
    return L.sage_kv_append(c or cache(), *a.values(), None)


def decode(L, c=None, **kw):
    a = dict(q=FAKE, qss=4 * 128, qsh=128, o=FAKE, lse=None, table=FAKE, M=4, lens=FAKE, S=2, Hq=4, window=64, sinks=0, weights=None,
             wstride=0, flags=4, ws=FAKE, size=1 << 30)
    a.update(kw)
    return L.sage_attn_paged_decode(c or cache(), *a.values(), None)


def evict(L, c=None, **kw):
    a = dict(table=FAKE, M=4, lens=FAKE, weights=FAKE, wstride=64, new_table=FAKE, M2=2, budget=20, first=2, last=3,
             new_lens=FAKE + 4096, new_weights=FAKE + 4096, kept=FAKE, S=2, ws=FAKE, size=1 << 30)
    a.update(kw)
    return L.sage_kv_evict(c or cache(), *a.values(), None)


CACHES = [dict(k=0), dict(v=FAKE + 8), dict(k_scale=FAKE), dict(k_scale=FAKE, v_scale=FAKE + 2), dict(pages=0), dict(page_size=0),
          dict(Hkv=0), dict(D=96), dict(ks=(4096, 2048, 4)), dict(vs=(-8, 2048, 128)), dict(page_size=1 << 29),
          dict(k_scale=FAKE, v_scale=FAKE, ks=(4352, 2176, 136))]     # 8-bit rows start on 16 bytes too


@pytest.mark.parametrize("bad", CACHES)
def test_cache_refusals(L, bad):
    for f in (append, decode, evict):
        assert f(L, cache(**bad)) == INVALID, f.__name__


@pytest.mark.parametrize("bad", [dict(ks=(2 * 16 * 128, 16 * 128, 64)), dict(vs=(0, 16 * 128, 128)), dict(vs=(2 * 16 * 128, 0, 128))])
def test_written_caches_have_no_rows_in_common(L, bad):
    for f in (append, evict):
        assert f(L, cache(**bad)) == INVALID, f.__name__


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=FAKE + 8), dict(pos=None), dict(pos=FAKE + 2), dict(counts=FAKE + 1), dict(S=0),
                                 dict(S=65536), dict(N=0), dict(flags=8), dict(table=None), dict(M=0), dict(weights=FAKE, ws=63),
                                 dict(ks=st(n=12)), dict(N=1 << 30)])
def test_append_refusals(L, bad):
    assert append(L, **bad) == INVALID


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=FAKE + 8), dict(qsh=4), dict(qss=-8), dict(o=None), dict(lse=FAKE + 2),
                                 dict(lens=None), dict(S=0), dict(Hq=3), dict(Hq=0), dict(window=0), dict(sinks=-1), dict(flags=0x20),
                                 dict(weights=FAKE, wstride=63), dict(weights=FAKE + 1, wstride=64), dict(ws=None, M=400),
                                 dict(ws=FAKE + 8, weights=FAKE, wstride=64),
                                 dict(table=FAKE + 2)])
def test_decode_refusals(L, bad):
    assert decode(L, **bad) == INVALID


def test_decode_workspace(L):
    need = bd.attn_paged_decode_workspace_size(3, 16, 2, 128, 100, 64, True)
    assert need > 3 * 16 * 6400 * 4
    c = cache(page_size=64)
    kw = dict(S=3, Hq=16, M=100, weights=FAKE, wstride=6400)
    assert decode(L, c, size=need - 1, **kw) == WORKSPACE
    assert 0 < bd.attn_paged_decode_workspace_size(3, 16, 2, 128, 100, 64) < need
    assert bd.attn_paged_decode_workspace_size(3, 16, 2, 128, 8, 64) == 0      # short: nothing is split
    for bad in ((0, 16, 2, 128, 1, 1), (1, 16, 3, 128, 1, 1), (1, 16, 2, 100, 1, 1), (1, 16, 2, 128, 0, 1), (1, 16, 2, 128, 1 << 16, 1 << 16)):
        assert bd.attn_paged_decode_workspace_size(*bad) == 0


@pytest.mark.parametrize("bad", [dict(lens=None), dict(weights=None), dict(new_table=None), dict(new_lens=None), dict(new_weights=None),
                                 dict(kept=FAKE + 2), dict(budget=0), dict(budget=33), dict(first=-1), dict(first=18), dict(last=-1),
                                 dict(M2=0), dict(wstride=63), dict(new_lens=FAKE), dict(new_weights=FAKE), dict(S=70000), dict(ws=None, M=2000, wstride=32000), dict(ws=FAKE + 64, M=2000, wstride=32000)])
def test_evict_refusals(L, bad):
    assert evict(L, **bad) == INVALID


def test_evict_workspace(L):
    need = bd.kv_evict_workspace_size(2, 2, 100, 1000)
    assert need >= 2 * 2 * 13 * 3 * 2048 * 4
    big = cache(page_size=1000, ks=(256000, 128000, 128), vs=(256000, 128000, 128))
    assert evict(L, big, M=100, wstride=100000, size=need - 1) == WORKSPACE
    assert bd.kv_evict_workspace_size(64, 2, 100, 1000) == 0 == bd.kv_evict_workspace_size(1, 1, 100, 100)
    for bad in ((0, 2, 1, 1), (2, 0, 1, 1), (2, 2, 0, 1), (2, 2, 1 << 16, 1 << 16)):
        assert bd.kv_evict_workspace_size(*bad) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch
    q = torch.zeros((1, 4, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        bd.sage_attn_window_fwd(q, q, q)
    with pytest.raises(TypeError):
        bd.sage_attn_window_fwd(q.float(), q, q)
    t = torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        bd.sage_attn_paged_decode(q[:, :, 0], q, q, t, t[0])
    with pytest.raises(ValueError):
        bd.sage_kv_append(q, q, q, q, t, t[0])
    with pytest.raises(ValueError):
        bd.sage_kv_evict(q, q, t, t[0], q, t, 4)


def test_more_blocks_than_a_launch_takes(L):
    big = dict(B=1 << 12, Hq=1 << 12, Hkv=1 << 12, N=1, D=64)            # 2^24 workgroups of 256
    assert fwd(L, **big) == INVALID
    assert bd.attn_window_bwd_workspace_size(*big.values()) == 0


@pytest.mark.parametrize("window,sinks", [(900, 100), (1, 999), (1, 5000), (999, 1), (1000, 1000)])
def test_window_that_reaches_the_sinks_is_no_window(L, window, sinks):
    # query 999 sees all of the keys 0 .. sinks - 1 and 1000 - window .. 999
    full = bd.attn_window_bwd_workspace_size(1, 4, 4, 1000, 128)
    assert bd.attn_window_bwd_workspace_size(1, 4, 4, 1000, 128, window, sinks) == full


def test_strides_whose_extent_overflows_are_refused(L):
    c = cache(ks=(1 << 40, 2048, 128), pages=(1 << 31) - 1)
    for f in (append, evict):
        assert f(L, c) == INVALID, f.__name__
