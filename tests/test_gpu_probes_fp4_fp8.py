"""Hardware semantics that the attention over an MXFP4 cache relies on: the register layout and scales of the
block-scaled 16x16x128 product of FP4 with FP8, and the scales of v_cvt_scalef32_pk_bf16_fp4 as E8M0 bytes."""
import ctypes
import os

import numpy as np
import pytest

from paper_2505_11594_amd import build as hb

import _more_lm as mo
from _gpu import torch_dev, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    torch_dev()
    assert os.path.exists(hb.PROBES_LIB), "libsage_probes.so is not built"
    L = ctypes.CDLL(hb.PROBES_LIB)
    vp = ctypes.c_void_p
    L.sage_probe_mfma_fp4_fp8.argtypes = [vp] * 6
    L.sage_probe_cvt_bf16_fp4.argtypes = [vp, vp, vp, ctypes.c_int, vp]
    return L


def e4m3(b):
    b = b.astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return np.where(b & 128, -v, v)


@pytest.mark.parametrize("spread", [0, 3])
def test_mfma_fp4_fp8_layout_and_scales(P, spread):
    """Products of few bits, whose sums are exact in fp32 in any order; all four places of a row's blocks and lanes."""
    import torch
    rng = np.random.default_rng(4 + spread)
    for rep in range(8):
        a = rng.integers(0, 256, (16, 64)).astype(np.uint8)
        b = (rng.integers(48, 64, (16, 128)) + 128 * rng.integers(0, 2, (16, 128))).astype(np.uint8)   # 2^-1 to 2^1, 4 bits
        sa, sb = (127 + rng.integers(-spread, spread + 1, (16, 4)) for _ in range(2))
        t = [torch.from_numpy(np.ascontiguousarray(x.astype(np.uint8))).cuda() for x in (a, sa, b, sb)]
        c = torch.zeros((16, 16), device="cuda")
        assert P.sage_probe_mfma_fp4_fp8(*[x.data_ptr() for x in t], c.data_ptr(), None) == 0
        torch.cuda.synchronize()
        av = mo.fp4_values(torch.from_numpy(a), torch.from_numpy(sa.astype(np.uint8))).numpy()
        bv = e4m3(b) * (2.0 ** (sb - 127.0)).repeat(32, -1)
        assert (c.cpu().numpy() == av @ bv.T).all(), rep


def test_cvt_bf16_fp4_takes_the_exponent_of_its_scale(P):
    """All codes by all scale bytes 1 to 253 as exponents of a float, exact in bf16."""
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8), 253)
    e = np.repeat(np.arange(1, 254, dtype=np.int64), 256)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy((e << 23).astype(np.int32)).cuda().view(torch.float32)
    y = torch.zeros(len(codes), dtype=torch.int32, device="cuda")
    assert P.sage_probe_cvt_bf16_fp4(c.data_ptr(), s.data_ptr(), y.data_ptr(), len(codes), None) == 0
    torch.cuda.synchronize()
    got = y.view(torch.bfloat16).view(-1, 2).double().cpu().numpy()
    v = np.array(mo.VALUES + [-x for x in mo.VALUES])
    want = np.stack([v[codes & 15], v[codes >> 4]], -1) * (2.0 ** (e - 127.0))[:, None]
    bad = (got != want).any(-1) & (np.abs(want).max(-1) < 2.0 ** 127.9)
    say("scales whose products differ: %s" % sorted(set(e[bad].tolist())))
    assert not bad.any()
