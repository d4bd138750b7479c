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


@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_more_tokens_than_a_launch_has_workgroups_for(in_place):
    """2^26 + 1000 tokens of one head, four a workgroup; pages only for the ends of both sequences."""
    n, R = (1 << 26) + 1000, 1 << 20
    new = torch.empty((n, 1, 64), dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    table = torch.full((2, 65), -1, dtype=torch.int32, device="cuda")
    table[0, 63], table[0, 64], table[1, 0] = 2, 0, 1
    k, v = (torch.zeros((3, 1, R, 64), dtype=BF16, device="cuda") for _ in "kv")
    pages = sa.make_pages(k=k, v=v, table=table, max_pages=65, page_rows=R, n_pages=3)
    rows = torch.tensor([[3], [9]], dtype=torch.int32, device="cuda")
    out = rows if in_place else torch.full_like(rows, -1)
    longest = n - 7
    cu = torch.tensor([0, longest, n], dtype=torch.int32, device="cuda")
    sa.seg_kv_paged_append(_cfg(2, 1, 1), pages, None, None, new, new, cu, n, longest, None, rows, None, out, _stream())
    assert out.tolist() == [[longest + 3], [16]]
    for pool in (k, v):
        assert torch.equal(pool[2, 0], new[63 * R - 3:64 * R - 3, 0])
        assert torch.equal(pool[0, 0, :longest + 3 - 64 * R], new[64 * R - 3:longest, 0]) and not pool[0, 0, longest + 3 - 64 * R:].any()
        assert torch.equal(pool[1, 0, 9:16], new[longest:, 0]) and not pool[1, 0, 16:].any() and not pool[1, 0, :9].any()


def test_eviction_of_more_windows_than_a_launch_has_workgroups_for():
    """32800 sequences of 128 heads, pages for the first and the last one."""
    B, H = 32800, 128
    k, v = (torch.randn((2, H, 4, 64), generator=torch.Generator().manual_seed(i)).to(BF16).cuda() for i in range(2))
    table = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[B - 1, 0] = 1, 0
    mass = torch.tensor([0.5, 2.0, 1.0, 9.0], device="cuda").expand(2, H, 4).contiguous()
    pos = torch.tensor([10, 11, 12, 13], dtype=torch.int32, device="cuda").expand(2, H, 4).contiguous()
    pages = sa.make_pages(k=k, v=v, table=table, max_pages=1, page_rows=4, n_pages=2, mass=mass, pos=pos)
    rows = torch.full((B, H), 3, dtype=torch.int32, device="cuda")
    want = [x.clone() for x in (k, v, mass, pos)]
    for x in want:
        x[:, :, 0] = x[:, :, 2]  # the heaviest two of three rows stay
    cfg = _cfg(B, H, H)
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pages, 4, 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_evict(cfg, pages, rows, 4, 2, 0, 0, rows, ws, need, _stream())
    assert (rows == 2).all()
    for x, y in zip((k, v, mass, pos), want):
        assert torch.equal(x, y)


def test_decode_of_more_heads_than_the_joining_launch_has_workgroups_for():
    """8200 sequences of 2048 query heads that share a page, a row or two each, in a table with room for windows that are cut."""
    B, H, g, R = 8200, 128, 16, 8224
    k, v = (torch.randn((1, H, R, 64), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda", dtype=BF16) for i in range(2))
    table = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    pages = sa.make_pages(k=k, v=v, table=table, max_pages=1, page_rows=R, n_pages=1)
    rows = torch.ones((B, H), dtype=torch.int32, device="cuda")
    rows[5], rows[6, 7] = 0, 100
    cfg = _cfg(B, H * g, H)
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, R)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    q = torch.ones((B, H * g, 64), dtype=BF16, device="cuda")
    out, lse = torch.full_like(q, float("nan")), torch.full((B, H * g), float("nan"), device="cuda")
    sa.seg_attn_decode_paged(cfg, pages, q, rows, R, out, lse, ws, need, stream=_stream())
    out = out.view(B, H, g, 64)
    one = v[0, :, 0][:, None].expand(H, g, 64)  # the only row, with the weight of one
    score = (k[0, :, 0].double().sum(-1) / 8)[:, None].expand(H, g)
    delta = 64 * 2.0 ** -24 * float(k[0, :, 0].double().abs().sum(-1).max()) / 8 + 2.0 ** -22 * (1 + float(score.abs().max()))
    some = torch.ones((B, H), dtype=torch.bool, device="cuda")
    some[5], some[6, 7] = False, False
    for b in range(0, B, 200):
        keep = some[b:b + 200]
        assert torch.equal(out[b:b + 200][keep], one.expand(200, H, g, 64)[keep])
        assert ((lse.view(B, H, g)[b:b + 200].double() - score)[keep].abs() <= delta).all()
    assert (out[5] == 0).all() and (lse[5] == -float("inf")).all()
    w = torch.softmax(k[0, 7, :100].double().sum(-1) / 8, 0)
    want = w @ v[0, 7, :100].double()
    assert ((out[6, 7].double() - want).abs() <= want.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -14 * v[0, 7, :100].double().abs().max()).all()
