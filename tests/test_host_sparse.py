"""CPU-only: what the operators for sparse attention over a paged cache refuse, before anything reaches a device."""
import ctypes

import pytest

import paper_2605_11744_amd as sa
from test_host_paged import BAD_PAGES, _cfg, _pages, _refused

P = 4096                                       # stand for device pointers: no call below gets as far as using them
K, T, U, R, G, S, W, Q, C, O, L = (P + (i << 24) for i in range(1, 12))


def pages(**kw):
    return _pages(**{**dict(k=K, v=K, table=T), **kw})


def blocks(**kw):
    return sa.make_blocks(**{**dict(block_rows=16, bounds=P + (20 << 24), scale=P + (21 << 24)), **kw})


def reserve(cfg=None, pg=None, **kw):
    a = dict(users=U, cu=P, total=9, longest=5, rows=R, granted=G, slots=S, ws=W, bytes=1 << 20, newest=False)
    a.update(kw)
    sa.seg_kv_paged_reserve(cfg or _cfg(), pg or pages(), a["users"], a["cu"], a["total"], a["longest"], a["rows"], a["granted"], a["slots"],
                            a["ws"], a["bytes"], newest_only=a["newest"])


def choose(cfg=None, pg=None, bl=None, **kw):
    a = dict(q=Q, cu=P, total=9, longest=5, rows=R, most=128, n=4, first=1, recent=1, chosen=C, ws=W, bytes=1 << 40)
    a.update(kw)
    sa.seg_kv_paged_choose(cfg or _cfg(), pg or pages(), bl or blocks(), a["q"], a["cu"], a["total"], a["longest"], a["rows"], a["most"], a["n"],
                           a["first"], a["recent"], a["chosen"], a["ws"], a["bytes"])


def attend(cfg=None, pg=None, bl=None, **kw):
    a = dict(q=Q, cu=P, total=9, longest=5, rows=R, most=128, chosen=C, n=4, out=O, lse=L, ws=W, bytes=1 << 22)
    a.update(kw)
    sa.seg_attn_paged_chosen(cfg or _cfg(), pg or pages(), bl or blocks(), a["q"], a["cu"], a["total"], a["longest"], a["rows"], a["most"],
                             a["chosen"], a["n"], a["out"], a["lse"], a["ws"], a["bytes"])


@pytest.mark.parametrize("bad", BAD_PAGES)
def test_pools_that_make_no_sense_are_refused(bad):
    bad = _pages(**bad)
    assert sa.seg_kv_paged_reserve_workspace_bytes(_cfg(), bad) == 0
    assert sa.seg_kv_paged_choose_workspace_bytes(_cfg(), bad, blocks(), 2, 100, 4) == 0
    assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), bad, blocks(), 2, 1, 100, 4) == 0
    _refused(reserve, None, bad)
    _refused(sa.seg_kv_paged_release, _cfg(), bad, U, R)
    _refused(sa.seg_kv_paged_summarize, _cfg(), bad, blocks(), None, R, 100)
    _refused(choose, None, bad)
    _refused(attend, None, bad)


@pytest.mark.parametrize("bad", [dict(fp32_check=True), dict(kv_policy=[1, 2], retrieved_capacity=8), dict(head_dim=96), dict(kv_policy=[1, 4])])
def test_configurations_without_a_paged_form_are_refused(bad):
    cfg = _cfg(**bad)
    assert sa.seg_kv_paged_reserve_workspace_bytes(cfg, pages()) == 0
    _refused(reserve, cfg)
    _refused(sa.seg_kv_paged_release, cfg, pages(), U, R)
    _refused(sa.seg_kv_paged_summarize, cfg, pages(), blocks(), None, R, 100)
    _refused(choose, cfg)
    _refused(attend, cfg)


BATCHES = [dict(total=-1), dict(total=0, cu=None), dict(total=0, longest=0), dict(total=0, longest=1 << 31), dict(longest=0), dict(total=4), dict(total=11), dict(total=1 << 31, longest=1 << 30), dict(cu=None), dict(cu=P + 2),
           dict(cu=None, total=2, longest=2)]


@pytest.mark.parametrize("bad", BATCHES)
def test_batches_that_make_no_sense_are_refused(bad):
    for call in (reserve, choose, attend):
        _refused(call, **bad)


@pytest.mark.parametrize("bad", [
    dict(users=None), dict(rows=None), dict(granted=None), dict(ws=None), dict(users=U + 2), dict(rows=R + 1), dict(granted=G + 2), dict(slots=S + 4),
    dict(ws=W + 128), dict(bytes=100), dict(users=T), dict(granted=R + 8), dict(slots=G), dict(users=P), dict(ws=T), dict(slots=R - 8), dict(granted=U + 32),
])
def test_reserve_refuses_buffers(bad):
    _refused(reserve, **bad)


def test_reserve_refuses_sizes():
    cfg, pg = _cfg(), pages()
    need = sa.seg_kv_paged_reserve_workspace_bytes(cfg, pg)
    assert need >= 4 * (2 + 1 + 9)
    _refused(reserve, bytes=need - 1)
    pg.per_head, pg.page_rows, pg.max_pages = 1, 1, 1 << 30  # two heads' entries of a sequence: 2^31
    assert sa.seg_kv_paged_reserve_workspace_bytes(cfg, pg) == 0
    for newest in (2, -1):
        status = sa.lib().seg_kv_paged_reserve(ctypes.byref(cfg), ctypes.byref(pages()), U, P, 9, 5, R, newest, G, S, W, 1 << 20, None)
        assert status == sa.SEGATTN_EINVAL


@pytest.mark.parametrize("users,rows", [(None, R), (U, None), (U + 1, R), (U, R + 2), (T, R), (R, R), (U, T), (R + 8, R)])
def test_release_refuses_buffers(users, rows):
    _refused(sa.seg_kv_paged_release, _cfg(), pages(), users, rows)


BAD_BLOCKS = [dict(block_rows=0), dict(block_rows=8), dict(block_rows=-16), dict(block_rows=24), dict(block_rows=64), dict(block_rows=1 << 30)]


@pytest.mark.parametrize("bad", BAD_BLOCKS + [dict(bounds=None), dict(scale=None), dict(bounds=P + 8)])
def test_blocks_that_make_no_sense_are_refused(bad):
    bl = blocks(**bad)
    _refused(sa.seg_kv_paged_summarize, _cfg(), pages(), bl, None, R, 100)
    _refused(choose, bl=bl)
    assert sa.seg_kv_paged_choose_workspace_bytes(_cfg(), pages(), bl, 2, 100, 4) == 0
    if "block_rows" in bad:
        _refused(attend, bl=bl)
        assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pages(), bl, 2, 1, 100, 4) == 0


def test_summarize_refuses_sizes_and_buffers():
    cfg, pg, bl = _cfg(), pages(), blocks()
    for rows_from, rows, most in ((None, None, 9), (None, R + 2, 9), (R + 1, R, 9), (None, R, 0), (None, R, 1 << 31), (bl.bounds, R, 9), (None, bl.scale, 9)):
        _refused(sa.seg_kv_paged_summarize, cfg, pg, bl, rows_from, rows, most)
    _refused(sa.seg_kv_paged_summarize, _cfg(kv_policy=[1, 0]), pg, bl, None, R, 9)
    _refused(sa.seg_kv_paged_summarize, cfg, pg, blocks(bounds=T), None, R, 9)
    _refused(sa.seg_kv_paged_summarize, cfg, pg, blocks(scale=blocks().bounds + 100), None, R, 9)


@pytest.mark.parametrize("bad", [
    dict(n=0), dict(n=4097), dict(first=-1), dict(recent=0), dict(recent=5), dict(first=4), dict(first=2 ** 31 - 1, recent=1), dict(most=0), dict(most=129),
    dict(q=None), dict(rows=None), dict(chosen=None), dict(ws=None), dict(q=Q + 8), dict(rows=R + 2), dict(chosen=C + 1), dict(ws=W + 16), dict(bytes=64),
    dict(chosen=Q), dict(chosen=R), dict(ws=C), dict(chosen=T), dict(chosen=P + (20 << 24)), dict(ws=P),
])
def test_choose_refuses_sizes_and_buffers(bad):
    _refused(choose, **bad)


def test_choose_refuses_heads():
    _refused(choose, _cfg(kv_policy=[0, 1]))
    _refused(choose, _cfg(n_q_heads=2 * 129))
    need = sa.seg_kv_paged_choose_workspace_bytes(_cfg(), pages(), blocks(), 9, 128, 4)
    assert need >= 9 * 8 * 4  # a key of every block for each token
    _refused(choose, bytes=need - 1)


@pytest.mark.parametrize("bad", [
    dict(n=0), dict(n=65537), dict(most=0), dict(most=129), dict(q=None), dict(rows=None), dict(chosen=None), dict(out=None), dict(lse=None), dict(ws=None),
    dict(q=Q + 8), dict(rows=R + 2), dict(chosen=C + 2), dict(out=O + 1), dict(lse=L + 2), dict(ws=W + 32), dict(bytes=0), dict(out=Q), dict(lse=O + 64),
    dict(out=R), dict(ws=Q), dict(lse=C), dict(out=T), dict(ws=O),
])
def test_attention_refuses_sizes_and_buffers(bad):
    _refused(attend, **bad)


def test_attention_refuses_heads_and_lists_beyond_31_bits():
    _refused(attend, _cfg(n_q_heads=2 * 129))
    assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(n_q_heads=2 * 128), pages(), blocks(), 9, 5, 128, 4) > 0
    pg = pages(page_rows=1 << 16, max_pages=1 << 10)
    assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pg, blocks(block_rows=1 << 16), 9, 5, 128, 30000) > 0
    assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pg, blocks(block_rows=1 << 16), 9, 5, 128, 32768) == 0
    for total, longest in ((-1, 1), (0, 0), (9, 0), (9, 4), (4, 5)):
        assert sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pages(), blocks(), total, longest, 128, 4) == 0


def test_a_step_of_one_sequence_has_room_for_its_parts():
    cfg, pg = _cfg(batch=1), pages(max_pages=1 << 12)
    need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pg, blocks(), 1, 1, 1 << 17, 256)
    assert need > 8 * (128 + 2) * 4
    _refused(attend, cfg, pg, total=1, longest=1, cu=None, most=1 << 17, n=256, bytes=need - 1)


def test_a_batch_without_tokens_has_nothing_to_be_done():
    """Choice and attention then write nothing, and need nothing of what belongs to tokens; what else is refused still is."""
    assert sa.seg_kv_paged_choose_workspace_bytes(_cfg(), pages(), blocks(), 0, 128, 4) > 0
    need = sa.seg_attn_paged_chosen_workspace_bytes(_cfg(), pages(), blocks(), 0, 5, 128, 4)
    assert need > 0
    choose(total=0, q=None, chosen=None)
    attend(total=0, q=None, chosen=None, out=None, lse=None, bytes=need)
    choose(total=0, q=R, chosen=T)  # an array of no elements shares nothing
    attend(total=0, out=T, lse=R)
    for bad in (dict(rows=None), dict(ws=None), dict(most=129), dict(bytes=0), dict(ws=T)):
        _refused(choose, total=0, **bad)
        _refused(attend, total=0, **bad)


def test_structure_has_the_layout_of_the_header():
    assert ctypes.sizeof(sa.segattn_blocks) == 4 + 4 + 2 * 8
