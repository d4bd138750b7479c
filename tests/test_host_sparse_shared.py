"""CPU-only: arrays of the pool that a call of the sparse attention must not write over."""
import pytest

import paper_2605_11744_amd as sa
from test_host_paged import _cfg, _refused
from test_host_sparse import C, L, O, P, R, W, attend, blocks, choose, pages

# 9 pages of 2 heads of 32 rows: 576 scale bytes, 2304 bytes of masses or positions
ROWS = 9 * 2 * 32
POOL = {"k_scale": ROWS, "v_scale": ROWS, "mass": 4 * ROWS, "pos": 4 * ROWS}


def _over(name, at, size):
    """A pool whose array `name` ends a few bytes into the buffer at `at`, or begins at its last ones."""
    apart = {x: P + ((30 + i) << 24) for i, x in enumerate(POOL)}
    for place in (at - POOL[name] + 4, at + size - 4):
        yield pages(e4m3=True, **{**apart, name: place})


@pytest.mark.parametrize("name", POOL)
def test_what_a_call_writes_is_not_an_array_of_the_pool(name):
    heads = 9 * 8
    for at, size in ((O, heads * 128 * 2), (L, heads * 4), (W, sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pages(), blocks(), 9, 5, 128, 4))):
        for pg in _over(name, at, size):
            _refused(attend, pg=pg)
    for at, size in ((C, 9 * 4 * 4), (W, sa.seg_kv_paged_choose_workspace_bytes(_cfg(), pages(), blocks(), 9, 128, 4))):
        for pg in _over(name, at, size):
            _refused(choose, pg=pg)
    bl = blocks()
    for at, size in ((bl.bounds, 9 * 2 * 2 * 2 * 128), (bl.scale, 9 * 2 * 2)):
        for pg in _over(name, at, size):
            _refused(sa.seg_kv_paged_summarize, _cfg(), pg, bl, None, R, 100)


def test_scales_are_not_looked_at_where_rows_are_bf16():
    """The fields are then nobody's.  (A batch without tokens: nothing is launched.)"""
    for call in (attend, choose):
        call(pg=pages(k_scale=W, v_scale=W), total=0)
        _refused(call, pg=pages(e4m3=True, k_scale=W, v_scale=P + (31 << 24)), total=0)
