"""CPU-only: what the operators around a paged cache refuse, before anything reaches a device."""
import ctypes

import pytest

import paper_2605_11744_amd as sa

P = 4096  # stands for a device pointer: no call below gets as far as using it
K = P + (1 << 20)  # and for another one


def _cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, seg_len=64, tail_len=16, kv_policy=[1, 2])
    base.update(kw)
    return sa.make_config(**base)


def _pages(**kw):
    base = dict(k=P, v=P, table=P, max_pages=4, page_rows=32, n_pages=9, mass=P, pos=P)
    base.update(kw)
    return sa.make_pages(**base)


def _rope(**kw):
    base = dict(theta=10000.0)
    base.update(kw)
    return sa.make_rope(**base)


def _refused(call, *args, **kw):
    with pytest.raises(sa.SegattnError) as e:
        call(*args, **kw)
    assert e.value.status == sa.SEGATTN_EINVAL


BAD_ROPES = [
    dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(rotary_dim=24), dict(rotary_dim=144),
    dict(rotary_dim=-16), dict(rotary_dim=8), dict(scaling=4), dict(scaling=-1), dict(scaling=sa.SEGATTN_ROPE_LINEAR, factor=0.0),
    dict(scaling=sa.SEGATTN_ROPE_LINEAR, factor=float("nan")), dict(magnitude=-1.0), dict(magnitude=float("inf")),
    dict(scaling=sa.SEGATTN_ROPE_BY_ROTATIONS, factor=2.0), dict(scaling=sa.SEGATTN_ROPE_BY_ROTATIONS, factor=2.0, trained_len=4096.0, low=4.0, high=4.0),
    dict(scaling=sa.SEGATTN_ROPE_BY_INDEX, factor=2.0, trained_len=4096.0, low=0.0, high=4.0),
    dict(scaling=sa.SEGATTN_ROPE_BY_INDEX, factor=2.0, trained_len=4096.0, low=1.0, high=4.0, theta=1.0),
    dict(inv_freq=[float("nan")] * 64), dict(inv_freq=[float("inf")] * 64),
]


@pytest.mark.parametrize("bad", BAD_ROPES)
def test_rotations_that_make_no_sense_are_refused(bad):
    _refused(sa.seg_rope_rotate, _cfg(), _rope(**bad), P, K, 5, P, K)
    _refused(sa.seg_kv_paged_append, _cfg(), _pages(), _rope(**bad), P, K, K, None, 2, 1, None, P, P, P)


@pytest.mark.parametrize("bad", [
    dict(q=None, k=None, q_out=None, k_out=None), dict(q_out=None), dict(q=None), dict(k_out=None), dict(rows=0), dict(rows=1 << 31),
    dict(q=P + 8), dict(k_out=P + 2), dict(q_stride=1000), dict(q_stride=1028), dict(k_out_stride=255), dict(pos0=P, pos=P),
    dict(pos0=P + 4), dict(pos=P + 4), dict(q_stride=2048), dict(k_stride=512),
])
def test_rotate_refuses_pointers_and_strides(bad):
    a = dict(q=P, k=K, rows=5, q_out=P, k_out=K)
    a.update(bad)
    _refused(sa.seg_rope_rotate, _cfg(), _rope(), a.pop("q"), a.pop("k"), a.pop("rows"), a.pop("q_out"), a.pop("k_out"), **a)


@pytest.mark.parametrize("bad", [
    dict(q_out=P + 16), dict(q_out=P - 16), dict(q_out=P + 5 * 2 * 2048 - 16), dict(k_out=P), dict(k_out=K + 512), dict(q_out=K - 16, k_out=K + 8192),
    dict(q_stride=2048, q_out_stride=4096), dict(q_out=P + 2 * 1008, q_stride=2048, q_out_stride=2048),
    dict(q_out=P - 2 * 1008, q_stride=2048, q_out_stride=2048), dict(k=P, k_out=P + 2 * 1024, q_stride=1280, q_out_stride=1280, k_stride=1280, k_out_stride=1264),
    dict(q_out=P + (1 << 16), k_out=P + (1 << 16) + 1024, k_out_stride=1024, q_out_stride=1024),
    dict(rows=1 << 29, q_stride=(1 << 32) - 8, q_out_stride=(1 << 32) - 8, q_out=P + 16, fp32=True),
])
def test_rotate_refuses_outputs_that_share_rows_with_something(bad):
    """Rows of 1024 and 256 channels; two sequences of five rows unless it says otherwise."""
    a = dict(q=P, k=K, rows=5, q_out=P, k_out=K)
    a.update(bad)
    _refused(sa.seg_rope_rotate, _cfg(), _rope(), a.pop("q"), a.pop("k"), a.pop("rows"), a.pop("q_out"), a.pop("k_out"), **a)


BAD_PAGES = [
    dict(k=None), dict(v=None), dict(table=None), dict(k=P + 8), dict(table=P + 2), dict(page_rows=0), dict(page_rows=-4), dict(n_pages=0),
    dict(max_pages=0), dict(max_pages=1 << 20, page_rows=1 << 11), dict(e4m3=True), dict(e4m3=True, k_scale=P),
    dict(row_stride=64, head_stride=4096, page_stride=8192), dict(row_stride=132, head_stride=8192, page_stride=16384),
    dict(row_stride=128, head_stride=4100, page_stride=8192), dict(row_stride=128, head_stride=4096, page_stride=0),
    dict(row_stride=128, head_stride=0, page_stride=8192), dict(row_stride=128, head_stride=-4096, page_stride=8192),
    dict(mass=P + 2), dict(pos=P + 1), dict(row_stride=128, head_stride=4096, page_stride=1 << 40),
    dict(row_stride=128, head_stride=4096, page_stride=1 << 39, n_pages=1 << 30),
]


@pytest.mark.parametrize("bad", BAD_PAGES)
def test_pools_that_make_no_sense_are_refused(bad):
    cfg, pages = _cfg(), _pages(**bad)
    assert sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, 100) == 0
    assert sa.seg_kv_paged_evict_workspace_bytes(cfg, pages, 100, 50) == 0
    _refused(sa.seg_attn_decode_paged, cfg, pages, P, P, 100, P, P, P, 1 << 40)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 100, 50, 10, 2, P, P, 1 << 40)
    _refused(sa.seg_kv_paged_append, cfg, pages, None, None, P, P, None, 2, 1, None, P, None, P)


def test_types_of_pages_and_layouts_outside_the_enums_are_refused():
    for field, value in (("type", 2), ("type", -1), ("per_head", 2), ("per_head", -1)):
        pages = _pages()
        setattr(pages, field, value)
        assert sa.seg_attn_decode_paged_workspace_bytes(_cfg(), pages, 100) == 0


@pytest.mark.parametrize("bad", [dict(fp32_check=True), dict(kv_policy=[1, 2], retrieved_capacity=8), dict(head_dim=96), dict(kv_policy=[1, 4])])
def test_configurations_without_a_paged_form_are_refused(bad):
    cfg = _cfg(**bad)
    assert sa.seg_attn_decode_paged_workspace_bytes(cfg, _pages(), 100) == 0
    _refused(sa.seg_kv_paged_append, cfg, _pages(), None, None, P, P, None, 2, 1, None, P, None, P)
    _refused(sa.seg_kv_paged_evict, cfg, _pages(), P, 100, 50, 10, 2, P, P, 1 << 40)


def test_append_refuses_what_it_cannot_place():
    ok = dict(q=P, k=K, v=K, cu=P, total=9, longest=5, pos0=P, rows=P, q_out=P, rows_out=P, rope=_rope())
    for bad in (dict(k=None), dict(v=None), dict(rows=None), dict(rows_out=None), dict(q_out=None), dict(q=None), dict(cu=None),
                dict(cu=None, total=2, longest=2), dict(total=4), dict(total=11), dict(longest=0), dict(total=1 << 31, longest=1 << 30),
                dict(rope=None, q_out=P + 16), dict(q=P + 2), dict(k=P + 8), dict(pos0=P + 4), dict(rows=P + 1), dict(rows_out=P + 4),
                dict(q_out=P + 256), dict(k=P), dict(v=P + 2 * 9 * 1024 - 16), dict(q=K, q_out=K, k=K - 2 * 9 * 256 + 16, v=P)):
        a = {**ok, **bad}
        _refused(sa.seg_kv_paged_append, _cfg(), _pages(), a["rope"], a["q"], a["k"], a["v"], a["cu"], a["total"], a["longest"], a["pos0"],
                 a["rows"], a["q_out"], a["rows_out"])


def test_decode_refuses_sizes_and_buffers():
    cfg, pages = _cfg(), _pages()
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, 128, True)
    assert need > sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, 128) > 0
    # scores: one PAST head, four query heads, 128 rows, two sequences
    assert need - sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, 128) == 2 * 4 * 128 * 4
    for rows in (0, -1, 129, 1 << 40):
        assert sa.seg_attn_decode_paged_workspace_bytes(cfg, pages, rows) == 0
        _refused(sa.seg_attn_decode_paged, cfg, pages, P, P, rows, P, P, P, 1 << 40)
    for i in range(5):  # q, rows, out, lse, workspace
        args = [P, P, P, P, P]
        args[i] = None
        _refused(sa.seg_attn_decode_paged, cfg, pages, args[0], args[1], 128, args[2], args[3], args[4], need, accumulate=True)
        args[i] = P + 1
        _refused(sa.seg_attn_decode_paged, cfg, pages, args[0], args[1], 128, args[2], args[3], args[4], need, accumulate=True)
    _refused(sa.seg_attn_decode_paged, cfg, pages, P, P, 128, P, P, P, need - 1, accumulate=True)
    _refused(sa.seg_attn_decode_paged, cfg, _pages(mass=None), P, P, 128, P, P, P, need, accumulate=True)
    _refused(sa.seg_attn_decode_paged, _cfg(kv_policy=[1, 1]), pages, P, P, 128, P, P, P, need, accumulate=True)
    assert sa.seg_attn_decode_paged_workspace_bytes(_cfg(n_q_heads=2 * 129), pages, 128) == 0
    assert sa.seg_attn_decode_paged_workspace_bytes(_cfg(n_q_heads=2 * 128), pages, 128) > 0


def test_evict_refuses_budgets_and_buffers():
    cfg, pages = _cfg(), _pages()
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pages, 128, 100)
    assert need > 0
    for rows, keep, recent, first in ((0, 100, 0, 0), (129, 100, 0, 0), (128, 0, 0, 0), (128, 100, 101, 0), (128, 100, 90, 11),
                                      (128, 100, -1, 0), (128, 100, 0, -1)):
        _refused(sa.seg_kv_paged_evict, cfg, pages, P, rows, keep, recent, first, P, P, 1 << 30)
    _refused(sa.seg_kv_paged_evict, cfg, _pages(mass=None), P, 128, 100, 10, 2, P, P, need)
    _refused(sa.seg_kv_paged_evict, cfg, _pages(pos=None), P, 128, 100, 10, 2, P, P, need)
    _refused(sa.seg_kv_paged_evict, _cfg(kv_policy=[1, 0]), pages, P, 128, 100, 10, 2, P, P, need)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 128, 100, 10, 2, P, P, need - 1)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 128, 100, 10, 2, P + 4, P, need)  # overlaps rows
    _refused(sa.seg_kv_paged_evict, cfg, pages, None, 128, 100, 10, 2, P, P, need)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 128, 100, 10, 2, None, P, need)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 128, 100, 10, 2, P, None, need)
    _refused(sa.seg_kv_paged_evict, cfg, pages, P, 128, 100, 10, 2, P, P + 128, need)


def test_structures_have_the_layout_of_the_header():
    assert ctypes.sizeof(sa.segattn_rope) == 8 + 3 * 4 + 4 + 5 * 8 + 8
    assert ctypes.sizeof(sa.segattn_pages) == 2 * 8 + 5 * 4 + 4 + 3 * 8 + 5 * 8
