"""What the attention over an MXFP4 cache relies on: v_cvt_scalef32_pk_bf16_fp4 takes an E8M0 byte as the exponent of its scale."""
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
    L.sage_probe_cvt_bf16_fp4.argtypes = [vp, vp, vp, ctypes.c_int, vp]
    return L


def test_cvt_bf16_fp4_takes_the_exponent_of_its_scale(P):
    """All codes by all scale bytes 0 to 253 as exponents of a float (0: 2^-127, no zero), exact in bf16."""
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8), 254)
    e = np.repeat(np.arange(254, dtype=np.int64), 256)
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
