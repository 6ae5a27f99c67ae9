"""Shapes that a caller hands to the binding may be lists, tuples or torch.Size."""
import types

import pytest

from paper_2505_11594_amd import binding as bd


def test_a_buffer_is_checked_against_any_sequence_of_sizes():
    import numpy as np
    import torch
    t, dev = torch.zeros(1, 2, 3, 4), types.SimpleNamespace(index=torch.zeros(1).get_device())
    for shape in ((1, 2, 3, 4), [1, 2, 3, 4], t.shape, np.array([1, 2, 3, 4]), (np.int64(1), 2, 3, 4)):
        bd._check_tensor(t, "out", shape, torch.float32, dev)
    for shape in ((1, 2, 3), [1, 2, 4, 3], t.shape[:3], [], np.array([1, 2, 3, 5])):
        with pytest.raises(ValueError):
            bd._check_tensor(t, "out", shape, torch.float32, dev)


@pytest.mark.gpu
def test_prequantized_attention_takes_its_shape_as_a_list():
    from _gpu import torch_dev
    torch = torch_dev()
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((1, 2, 256, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    codes = [bd.sage_quant_fp4(x, role)[:2] for x, role in ((q, bd.SAGE_ROLE_Q), (k, bd.SAGE_ROLE_K), (v, bd.SAGE_ROLE_V))]
    want = bd.sage_attn_fp4_fwd_prequant(*codes, (1, 2, 256, 64))
    out = torch.zeros_like(want)
    for shape in ([1, 2, 256, 64], q.shape):
        assert torch.equal(bd.sage_attn_fp4_fwd_prequant(*codes, shape), want)
        assert bd.sage_attn_fp4_fwd_prequant(*codes, shape, out=out.zero_()) is out and torch.equal(out, want)
    with pytest.raises(ValueError):
        bd.sage_attn_fp4_fwd_prequant(*codes, [1, 2, 256, 64], out=out[:, :1])
