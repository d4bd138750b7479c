"""CPU-only: the sizes up to which the paged operators go, as the header states them."""
import pytest

import paper_2605_11744_amd as sa

P = 4096  # stands for a device pointer


def _pages(**kw):
    base = dict(k=P, v=P, table=P, max_pages=1, page_rows=1 << 22, n_pages=9, mass=P, pos=P)
    base.update(kw)
    return sa.make_pages(**base)


def _cfg(batch, hq, hkv):
    return sa.make_config(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=64, seg_len=64, tail_len=16, kv_policy=[2] * hkv)


@pytest.mark.parametrize("batch,hq,hkv,rows,fits", [
    ((1 << 24) - 1, 1, 1, 32, True), (1 << 24, 1, 1, 32, False),          # B * Hkv
    ((1 << 23) - 1, 128, 1, 32, True), (1 << 23, 128, 1, 32, False),      # B * Hq
    (1 << 14, 8, 1, 32 * ((1 << 17) - 2), True), (1 << 14, 8, 1, 32 * ((1 << 17) - 2) + 1, False),  # tiles
])
def test_decode_goes_up_to_what_the_header_says(batch, hq, hkv, rows, fits):
    cfg = _cfg(batch, hq, hkv)
    assert (sa.seg_attn_decode_paged_workspace_bytes(cfg, _pages(), rows) > 0) == fits
    if not fits:
        with pytest.raises(sa.SegattnError) as e:
            sa.seg_attn_decode_paged(cfg, _pages(), P, P, rows, P, P, P, 1 << 45)
        assert e.value.status == sa.SEGATTN_EINVAL


@pytest.mark.parametrize("batch,fits", [((1 << 24) - 1, True), (1 << 24, False)])
def test_eviction_goes_up_to_what_the_header_says(batch, fits):
    assert (sa.seg_kv_paged_evict_workspace_bytes(_cfg(batch, 1, 1), _pages(), 32, 16) > 0) == fits


@pytest.mark.parametrize("strides,fits", [
    (dict(row_stride=1 << 25, head_stride=1 << 39, page_stride=(1 << 40) - 8), True), (dict(row_stride=(1 << 25) + 8, head_stride=1 << 39, page_stride=1 << 39), False),
    (dict(row_stride=64, head_stride=1 << 40, page_stride=1 << 39), False), (dict(row_stride=64, head_stride=64, page_stride=1 << 40), False),
    (dict(row_stride=64, head_stride=64, page_stride=1 << 39, n_pages=1 << 22), False),
])
def test_pools_go_up_to_what_the_header_says(strides, fits):
    pages = _pages(**{"page_rows": 32, **strides})
    assert (sa.seg_attn_decode_paged_workspace_bytes(_cfg(2, 2, 2), pages, 32) > 0) == fits
