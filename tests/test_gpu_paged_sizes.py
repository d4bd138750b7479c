"""Calls whose workgroups do not fit one launch (fewer than 2^32 threads in a dimension), on tensors of few channels so that the
sizes stay within some ten GB."""
import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _cfg(batch, hq, hkv):
    return sa.make_config(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=64, seg_len=64, tail_len=16, kv_policy=[2] * hkv)


def test_rotation_of_more_tokens_than_a_launch_has_workgroups_for():
    """2^28 + 1000 tokens of one head, 16 a workgroup: 34 GB, in place."""
    n = (1 << 28) + 1000
    x = torch.empty((n, 1, 64), dtype=BF16, device="cuda")
    for a in range(0, n, 1 << 26):
        x[a:a + (1 << 26)].normal_(generator=torch.Generator(device="cuda").manual_seed(a))
    parts = [(0, 100), ((1 << 28) - 60, (1 << 28) + 60), (n - 50, n), (123456789, 123456800)]
    before = [x[a:z].clone() for a, z in parts]
    sa.seg_rope_rotate(_cfg(1, 1, 1), sa.make_rope(theta=10000.0), x, None, n, x, None, stream=_stream())
    for (a, z), b in zip(parts, before):
        want, size = ref.turned(b.double().cpu(), range(a, z), dict(theta=10000.0))
        assert ((x[a:z].double().cpu() - want).abs() <= want.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + size * 2.0 ** -20).all(), a
