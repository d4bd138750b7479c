"""Row counts that an eviction leaves where heads hold more than the call was promised."""
import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref
from paged_ref import Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_rows,keep", [(100, 60), (50, 60), (60, 60), (1, 60), (100, 10 ** 12), (10, 2 ** 31)])
@pytest.mark.parametrize("in_place", [False, True])
def test_counts_end_at_the_budget_whatever_was_promised(max_rows, keep, in_place):
    pool = Pool(batch=4, hkv=2, d=64, page_rows=16, max_pages=10).fill([150, 61, 60, 3])
    pool.rows[3, 0] = -2
    cfg = sa.make_config(batch=4, n_q_heads=2, n_kv_heads=2, head_dim=64, seg_len=64, tail_len=16, kv_policy=[2, 1])
    want = pool.rows.clone()
    want[:, 0].clamp_(max=min(keep, 2 ** 31 - 1))
    before = pool.state()
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pool.pages(), max_rows, keep)
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), pool.rows if in_place else torch.full_like(pool.rows, 77)
    sa.seg_kv_paged_evict(cfg, pool.pages(), pool.rows, max_rows, keep, 8, 2, out, ws, need, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out, want)
    if max_rows <= keep:
        for x in before:
            if x != "rows":
                assert torch.equal(ref.bits(getattr(pool, x)), ref.bits(before[x])), x
