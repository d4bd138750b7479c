"""fp32 outputs of the paged decode have the accuracy of fp32, not that of a rounded weight."""
import math

import pytest
import torch

import paper_2605_11744_amd as sa

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", [64, 8192], ids=["whole", "cut"])
@pytest.mark.parametrize("page_rows,e4m3", [(32, False), (16, False), (32, True)])
def test_a_weight_keeps_24_bits(d, room, page_rows, e4m3):
    """Two rows: one with score 0 and values 0, one with score -s and values 1, so that the output is e^-s / (1 + e^-s).  The
    scores are exact (one product of each sum is not zero).  What is rounded: log2(e) and its product with the score (2 half
    steps of 1.5 at most, times ln 2: 2.1 * 2^-24 of the weight), the exponential (2^-23), the sum, the reciprocal and the product
    with it (half a step each, 2^-23 for the reciprocal): below 2^-21 of the output; 2^-20 is allowed.  A weight rounded to two
    bf16 would be off by up to 2^-16."""
    B, hq = 40, 16
    s = torch.linspace(0.004, 1.0, B * hq, dtype=torch.float64).to(BF16).view(B, hq)
    q = torch.zeros((B, hq, d), dtype=BF16)
    q[..., 5] = -s
    k, v = (torch.zeros((1, 1, page_rows, d), dtype=BF16) for _ in "kv")
    k[0, 0, 1, 5], v[0, 0, 1] = 1.0, 1.0
    if e4m3:
        k, v = (x.to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
    k, v = k.cuda(), v.cuda()
    scale = torch.full((1, 1, page_rows), 127, dtype=torch.uint8, device="cuda")
    table = torch.zeros((B, room // page_rows), dtype=torch.int32, device="cuda")
    pages = sa.make_pages(k=k, v=v, table=table, max_pages=room // page_rows, page_rows=page_rows, n_pages=1, e4m3=e4m3, k_scale=scale, v_scale=scale)
    cfg = sa.make_config(batch=B, n_q_heads=hq, n_kv_heads=1, head_dim=d, seg_len=64, tail_len=0, kv_policy=[2], scale=1.0, out_fp32=True)
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, room)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    rows = torch.full((B, 1), 2, dtype=torch.int32, device="cuda")
    out, lse = torch.empty((B, hq, d), device="cuda"), torch.empty((B, hq), device="cuda")
    sa.seg_attn_decode_paged(cfg, pages, q.cuda(), rows, room, out, lse, ws, need, stream=torch.cuda.current_stream().cuda_stream)
    e = (-s.double()).exp()
    want = (e / (1 + e))[..., None]
    err = ((out.double().cpu() - want) / want).abs().max()
    assert err <= 2.0 ** -20, f"2^{math.log2(err):.2f}"
    assert ((lse.double().cpu() - (1 + e).log()).abs() <= 2.0 ** -21).all()
