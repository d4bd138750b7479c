"""8-bit rows at the ends of the range, from append to decode."""
import math

import pytest
import torch

import paper_2605_11744_amd as sa
from paged_ref import Pool

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# element and what the decode step makes of a row that holds nothing else: multiples of 2^120 that bf16 holds
TOP = [(192, 192), (239, 240), (240, 240), (247, 240), (248, math.inf), (255, math.inf), (-247, -240), (-248, -math.inf)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", [64, 8192], ids=["whole", "cut"])
@pytest.mark.parametrize("out_fp32", [False, True])
def test_the_largest_rows_come_back(d, room, out_fp32):
    B = len(TOP)
    pool = Pool(batch=B, hkv=1, d=d, page_rows=32, max_pages=room // 32, e4m3=True, spare=0)
    v = torch.tensor([x * 2.0 ** 120 for x, _ in TOP], dtype=torch.float64).to(BF16)
    assert v.double().tolist() == [x * 2.0 ** 120 for x, _ in TOP]
    v = v.view(B, 1, 1).expand(B, 1, d).contiguous().cuda()
    k = torch.zeros_like(v)
    cfg = sa.make_config(batch=B, n_q_heads=1, n_kv_heads=1, head_dim=d, seg_len=64, tail_len=0, kv_policy=[2], out_fp32=out_fp32)
    st = torch.cuda.current_stream().cuda_stream
    sa.seg_kv_paged_append(cfg, pool.pages(), None, None, k, v, None, B, 1, None, pool.rows, None, pool.rows, st)
    out, lse = torch.empty((B, 1, d), dtype=torch.float32 if out_fp32 else BF16, device="cuda"), torch.empty((B, 1), device="cuda")
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), room)
    sa.seg_attn_decode_paged(cfg, pool.pages(), torch.ones_like(k), pool.rows, room, out, lse, torch.empty(need, dtype=torch.uint8, device="cuda"), need, stream=st)
    assert (lse == 0).all()
    for b, (_, want) in enumerate(TOP):
        got = out[b, 0].double()
        if math.isinf(want):
            assert not got.isfinite().any()  # infinite, or NaN where parts of a weight of zero meet it
        else:
            assert (got == want * 2.0 ** 120).all(), b


@pytest.mark.parametrize("d", [64, 128])
def test_the_smallest_rows_come_back(d):
    """Elements below 448 * 2^-119 share the scale 2^-119 (steps of 2^-128, denormal in bf16): within half a step of e4m3,
    and what the products flush, 2^-126 at most."""
    x = torch.tensor([2.0 ** -100, 2.0 ** -112, 2.0 ** -118, 1.5 * 2.0 ** -121, 2.0 ** -126, 0.0], dtype=torch.float64)
    B = len(x)
    pool = Pool(batch=B, hkv=1, d=d, page_rows=32, max_pages=2, e4m3=True, spare=0)
    v = x.to(BF16).view(B, 1, 1).expand(B, 1, d).contiguous().cuda()
    cfg = sa.make_config(batch=B, n_q_heads=1, n_kv_heads=1, head_dim=d, seg_len=64, tail_len=0, kv_policy=[2], out_fp32=True)
    st = torch.cuda.current_stream().cuda_stream
    sa.seg_kv_paged_append(cfg, pool.pages(), None, None, torch.zeros_like(v), v, None, B, 1, None, pool.rows, None, pool.rows, st)
    out, lse = torch.empty((B, 1, d), device="cuda"), torch.empty((B, 1), device="cuda")
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), 64)
    sa.seg_attn_decode_paged(cfg, pool.pages(), torch.ones_like(v), pool.rows, 64, out, lse, torch.empty(need, dtype=torch.uint8, device="cuda"), need, stream=st)
    want = x.view(B, 1, 1)
    assert ((out.double().cpu() - want).abs() <= want * 2.0 ** -4 + 2.0 ** -129 + 2.0 ** -126).all()
