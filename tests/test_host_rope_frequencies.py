"""CPU-only: a list of frequencies has one per turned pair; the library is never handed a shorter one."""
import ctypes

import pytest

import paper_2605_11744_amd as sa
import paper_2605_11744_amd.binding as binding

P, K = 4096, 4096 + (1 << 20)  # stand for device pointers


class _Recorder:
    """Stands for the library and notes its calls."""

    def __init__(self):
        self.calls = []

    def segattn_strerror(self, status):
        return b"refused"

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or sa.SEGATTN_OK


@pytest.fixture
def calls(monkeypatch):
    recorder = _Recorder()
    monkeypatch.setattr(binding, "lib", lambda: recorder)
    return recorder.calls


def _both(d, **rope):
    cfg = sa.make_config(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=d, seg_len=64, tail_len=16, kv_policy=[1, 2])
    r = sa.make_rope(theta=10000.0, **rope)
    pages = sa.make_pages(k=P, v=P, table=P, max_pages=4, page_rows=32, n_pages=9)
    return (lambda: sa.seg_rope_rotate(cfg, r, P, None, 5, P, None),
            lambda: sa.seg_kv_paged_append(cfg, pages, r, P, K, K, None, 2, 1, None, P, P, P))


@pytest.mark.parametrize("d,rotary,n", [(128, 0, 32), (128, 0, 0), (128, 0, 65), (128, 64, 64), (128, 64, 16), (64, 0, 31), (64, 32, 17)])
def test_lists_of_another_length_never_reach_the_library(calls, d, rotary, n):
    for call in _both(d, rotary_dim=rotary, inv_freq=[0.5] * n):
        with pytest.raises(sa.SegattnError) as e:
            call()
        assert e.value.status == sa.SEGATTN_EINVAL
    assert calls == []


@pytest.mark.parametrize("d,rotary,n", [(128, 0, 64), (128, 64, 32), (64, 0, 32), (64, 16, 8), (64, 48, None)])
def test_lists_of_the_pairs_length_do(calls, d, rotary, n):
    for call in _both(d, rotary_dim=rotary, inv_freq=[0.5] * n if n else None):
        call()
    assert calls == ["seg_rope_rotate", "seg_kv_paged_append"]


def test_a_structure_filled_by_hand_is_the_callers_business(calls):
    """Only make_rope knows a length; a pointer that a program sets itself is passed on."""
    cfg = sa.make_config(batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, seg_len=64, tail_len=16, kv_policy=[1, 2])
    freq = (ctypes.c_double * 32)(*[0.5] * 32)
    rope = sa.segattn_rope(10000.0, 0, 0, sa.SEGATTN_ROPE_PLAIN, 1.0, 0.0, 0.0, 0.0, 0.0, ctypes.cast(freq, ctypes.POINTER(ctypes.c_double)))
    sa.seg_rope_rotate(cfg, rope, P, None, 5, P, None)
    assert calls == ["seg_rope_rotate"]
