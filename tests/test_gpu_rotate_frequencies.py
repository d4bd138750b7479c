"""Frequencies given as a list: nothing else of the rotation's description that forms frequencies is looked at."""
import ctypes
import math

import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", [dict(theta=0.0), dict(theta=-1.0), dict(theta=math.nan), dict(theta=math.inf), dict(theta=1.0, scaling=sa.SEGATTN_ROPE_BY_INDEX),
                                  dict(theta=1e4, scaling=sa.SEGATTN_ROPE_LINEAR, factor=0.0), dict(theta=1e4, scaling=99)], ids=str)
def test_a_list_stands_for_itself(rest):
    freq = [1.0 / (i + 1) for i in range(32)]
    cfg = sa.make_config(batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, seg_len=64, tail_len=16, kv_policy=[1, 1])
    x = torch.randn((50, 2, 64), generator=torch.Generator().manual_seed(1)).cuda()
    y = torch.empty_like(x)
    sa.seg_rope_rotate(cfg, sa.make_rope(inv_freq=freq, **rest), x, None, 50, y, None, fp32=True, stream=torch.cuda.current_stream().cuda_stream)
    want, size = ref.turned(x.double().cpu(), range(50), dict(theta=1.0, inv_freq=freq))
    assert ((y.double().cpu() - want).abs() <= want.abs() * 2.0 ** -24 + size * 2.0 ** -20).all()


def test_a_structure_that_holds_nothing_but_a_list():
    freq = (ctypes.c_double * 32)(*[0.25] * 32)
    rope = sa.segattn_rope()
    rope.inv_freq = ctypes.cast(freq, ctypes.POINTER(ctypes.c_double))
    cfg = sa.make_config(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, seg_len=64, tail_len=16, kv_policy=[1])
    x = torch.zeros((3, 1, 64), device="cuda")
    x[..., :32] = 1.0
    y = torch.empty_like(x)
    sa.seg_rope_rotate(cfg, rope, x, None, 3, y, None, fp32=True, stream=torch.cuda.current_stream().cuda_stream)
    for t in range(3):
        assert abs(float(y[t, 0, 0]) - math.cos(t / 4)) <= 2.0 ** -20 and abs(float(y[t, 0, 32]) - math.sin(t / 4)) <= 2.0 ** -20
