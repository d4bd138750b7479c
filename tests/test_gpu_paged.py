"""The operators around a paged cache against their definitions in 64 bits (paged_ref.py)."""
import math

import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref
from paged_ref import Pool

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _cfg(pool, hq, policy=None, seg=64, tail=16, **kw):
    return sa.make_config(batch=pool.B, n_q_heads=hq, n_kv_heads=pool.H, head_dim=pool.D, seg_len=seg, tail_len=tail,
                          kv_policy=policy or [2] * pool.H, **kw)


# ---- append ----------------------------------------------------------------------------------------
def _append_reference(pool, k, v, cu, pos0, rope):
    """The state that an append leaves, and where new key rows lie with their exact values and error sizes."""
    s = {x: y.cpu().clone() for x, y in pool.state().items()}
    keys = []
    for b in range(pool.B):
        m = cu[b + 1] - cu[b]
        if m == 0:
            continue
        at = torch.arange(m) + pos0[b]
        kk, vv = k[cu[b]:cu[b + 1]].to(torch.float64).cpu(), v[cu[b]:cu[b + 1]].to(torch.float64).cpu()
        size = torch.zeros_like(kk)
        if rope:
            kk, size = ref.turned(kk, at, rope)
        for h in range(pool.H):
            held = int(s["rows"][b, h])
            for i in range(m):
                row = held + i
                if row >= pool.max_pages * pool.R:
                    continue
                (page,), hh, (r,) = pool.place(b, h, [row])
                if page < 0:
                    continue
                if pool.e4m3:
                    (s["v"][page, hh, r],), (s["v_scale"][page, hh, r],) = ref.e4m3_rows(vv[i, h][None])
                else:
                    s["v"][page, hh, r] = vv[i, h].to(BF16)
                keys.append(((int(page), hh, int(r)), kk[i, h], size[i, h]))
                if "pos" in s:
                    s["pos"][page, hh, r] = int(at[i])
                if "mass" in s:
                    s["mass"][page, hh, r] = 0.0
            s["rows"][b, h] = min(held + m, pool.max_pages * pool.R)
    return s, keys


def _check_append(pool, want, keys, rope):
    got = pool.state()
    for x in got:
        if x not in ("k", "k_scale"):
            assert torch.equal(ref.bits(got[x]), ref.bits(want[x])), x
    k, scale = got["k"].cpu(), got["k_scale"].cpu() if pool.e4m3 else None
    for at, exact, size in keys:
        if not rope and not pool.e4m3:
            assert torch.equal(ref.bits(k[at]), ref.bits(exact.to(BF16)))
        elif pool.e4m3:
            s = 2.0 ** (int(scale[at]) - 127)
            most = float(exact.abs().max())
            assert most * (1 - 2.0 ** -18) <= 448 * s and (most * (1 + 2.0 ** -18) > 224 * s or s == 1.0)
            err = (k[at].view(torch.float8_e4m3fn).double() * s - exact).abs()
            # half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below 2^-6), and the turning's own error
            assert (err <= exact.abs() * 2.0 ** -4 + 2.0 ** -10 * s + size * 2.0 ** -19).all()
        else:
            assert ((k[at].double() - exact).abs() <= exact.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + size * 2.0 ** -20).all()
        k[at] = want["k"][at]  # the rest has to be as it was
        if pool.e4m3:
            scale[at] = want["k_scale"][at]
    assert torch.equal(ref.bits(k), ref.bits(want["k"]))
    if pool.e4m3:
        assert torch.equal(scale, want["k_scale"])


APPENDS = [
    dict(page_rows=16), dict(page_rows=1, max_pages=90), dict(page_rows=5, per_head=True), dict(page_rows=32, token_major=True, d=64),
    dict(page_rows=64, e4m3=True), dict(page_rows=7, e4m3=True, per_head=True, d=64), dict(page_rows=24, e4m3=True, token_major=True),
    dict(page_rows=8, mass=False, pos=False),
]


@pytest.mark.parametrize("kind", APPENDS, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
@pytest.mark.parametrize("rope", [None, dict(theta=10000.0), dict(theta=10000.0, rotary_dim=32, interleaved=True, magnitude=1.5)],
                         ids=["as_is", "turned", "part"])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_ragged_prompts(kind, rope, in_place):
    kind = {"max_pages": 12, "d": 128, **kind}
    hq, hkv = 6, 3
    pool = Pool(batch=4, hkv=hkv, **kind, seed=2).fill([[3, 0, 9], 0, 17, [1, 2, 3]])
    m = [19, 0, 1, 33]
    cu = [sum(m[:i]) for i in range(5)]
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn((cu[-1], h, pool.D), generator=g).to(BF16).cuda() for h in (hq, hkv, hkv))
    pos0 = torch.tensor([5, 0, 90000, 123], dtype=torch.int64)
    want, keys = _append_reference(pool, k, v, cu, pos0.tolist(), rope)
    rows_out = pool.rows if in_place else torch.full_like(pool.rows, -5)
    before = pool.rows.clone()
    q_out = (q if in_place else torch.empty_like(q)) if rope else None
    q_in = q.clone()
    sa.seg_kv_paged_append(_cfg(pool, hq), pool.pages(), sa.make_rope(**rope) if rope else None, q if rope else None, k, v,
                           torch.tensor(cu, dtype=torch.int32, device="cuda"), cu[-1], max(m), pos0.cuda(), pool.rows, q_out, rows_out, _stream())
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(pool.rows, before)
        pool.rows = rows_out
    _check_append(pool, want, keys, rope)
    if rope:
        at = torch.cat([torch.arange(x) + p for x, p in zip(m, pos0)])
        exact, size = ref.turned(q_in.to(torch.float64).cpu(), at, rope)
        assert ((q_out.double().cpu() - exact).abs() <= exact.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + size * 2.0 ** -20).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("named", [False, True], ids=["one_each", "cu_seqlens"])
def test_append_of_a_generation_step(e4m3, named):
    pool = Pool(batch=5, hkv=2, d=128, page_rows=16, max_pages=4, e4m3=e4m3).fill([0, 15, 16, [63, 64], 40])
    rope, hq = dict(theta=500000.0), 8
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((5, h, 128), generator=g).to(BF16).cuda() for h in (hq, 2, 2))
    pos0 = torch.tensor([0, 15, 160, 64, 400000], dtype=torch.int64)
    want, keys = _append_reference(pool, k, v, list(range(6)), pos0.tolist(), rope)
    cu = torch.arange(6, dtype=torch.int32, device="cuda") if named else None
    sa.seg_kv_paged_append(_cfg(pool, hq), pool.pages(), sa.make_rope(**rope), q, k, v, cu, 5, 1, pos0.cuda(), pool.rows, q, pool.rows, _stream())
    torch.cuda.synchronize()
    _check_append(pool, want, keys, rope)  # a full table (64 rows): the row is dropped, the count stays


def test_append_of_a_long_prompt_uses_many_workgroups():
    pool = Pool(batch=2, hkv=2, d=64, page_rows=32, max_pages=700, mass=False).fill([3, 100])
    n = 21000
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((n, 2, 64), generator=g).to(BF16).cuda() for _ in "kv")
    cu = torch.tensor([0, 20000, n], dtype=torch.int32, device="cuda")
    sa.seg_kv_paged_append(_cfg(pool, 4), pool.pages(), None, None, k, v, cu, n, 20000, None, pool.rows, None, pool.rows, _stream())
    assert pool.rows.tolist() == [[20003] * 2, [1100] * 2]
    for b, (lo, a, z) in enumerate(((3, 0, 20000), (100, 20000, n))):
        for h in range(2):
            page, hh, r = pool.place(b, h, torch.arange(lo, lo + z - a))
            assert torch.equal(pool.k[page.cuda(), hh, r.cuda()], k[a:z, h]) and torch.equal(pool.v[page.cuda(), hh, r.cuda()], v[a:z, h])
            assert torch.equal(pool.pos[page.cuda(), hh, r.cuda()].cpu(), torch.arange(z - a, dtype=torch.int32))


def test_append_leaves_rows_without_a_page_out():
    pool = Pool(batch=2, hkv=1, d=64, page_rows=4, max_pages=3)
    pool.table[0, 1], pool.table[1, 0] = -1, pool.n_pages
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((20, 1, 64), generator=g).to(BF16).cuda() for _ in "kv")
    cu = [0, 9, 20]
    want, keys = _append_reference(pool, k, v, cu, [0, 0], None)
    assert len(keys) == 9 - 4 + 11 - 4
    sa.seg_kv_paged_append(_cfg(pool, 1), pool.pages(), None, None, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 20, 11, None,
                           pool.rows, None, pool.rows, _stream())
    _check_append(pool, want, keys, None)
    # twelve more: behind the tables' ends
    want, keys = _append_reference(pool, k, v, [0, 10, 20], [0, 0], None)
    sa.seg_kv_paged_append(_cfg(pool, 1), pool.pages(), None, None, k, v, torch.tensor([0, 10, 20], dtype=torch.int32, device="cuda"), 20, 10, None,
                           pool.rows, None, pool.rows, _stream())
    assert pool.rows.tolist() == [[12], [12]]
    _check_append(pool, want, keys, None)


def test_e4m3_rows_of_every_magnitude():
    """Zeros, one large element among small ones, the type's extremes, values between two steps (to even), infinities and NaN."""
    pool = Pool(batch=1, hkv=1, d=64, page_rows=16, max_pages=1, e4m3=True)
    x = torch.zeros((9, 64), dtype=torch.float64)
    x[1, 0] = 448.0
    x[2, :3] = torch.tensor([1000.0, 0.001, -0.5])
    x[3] = torch.arange(64) * 2.0 ** -130
    x[4] = 3.3e38
    x[5] = (torch.arange(64) - 32) / 16.0 * 0.53125  # steps' midpoints among them
    x[6, :4] = torch.tensor([math.inf, -math.inf, math.nan, 5.0])
    x[7] = 449.0
    x[8] = torch.randn(64, generator=torch.Generator().manual_seed(2)) * 1e-4
    k = x.to(BF16).cuda().view(9, 1, 64)
    sa.seg_kv_paged_append(_cfg(pool, 1), pool.pages(), None, None, k, k, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), 9, 9, None,
                           pool.rows, None, pool.rows, _stream())
    want, scale = ref.e4m3_rows(k[:, 0].double().cpu())
    page, _, r = pool.place(0, 0, range(9))
    for got, s in ((pool.k, pool.k_scale), (pool.v, pool.v_scale)):
        assert s[page, 0, r].tolist() == scale.tolist()
        a, b = got[page, 0, r].cpu().view(torch.float8_e4m3fn).float(), want.view(torch.float8_e4m3fn).float()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())


# ---- decode ----------------------------------------------------------------------------------------
def _decode(pool, hq, lengths, *, policy=None, seg=64, tail=16, out_fp32=True, accumulate=False, max_rows=None, scale=0.0, q=None, seed=9):
    policy = policy or [2] * pool.H
    cfg = _cfg(pool, hq, policy, seg, tail, out_fp32=out_fp32, scale=scale)
    if q is None:
        q = torch.randn((pool.B, hq, pool.D), generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()
    out = torch.full((pool.B, hq, pool.D), float("nan"), dtype=torch.float32 if out_fp32 else BF16, device="cuda")
    lse = torch.full((pool.B, hq), float("nan"), device="cuda")
    most = max_rows or pool.max_pages * pool.R
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), most, accumulate)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    before = pool.mass.double().cpu() if accumulate else None
    sa.seg_attn_decode_paged(cfg, pool.pages(), q, pool.rows, most, out, lse, ws, need, accumulate=accumulate, stream=_stream())
    torch.cuda.synchronize()
    want, want_lse, weights, most_s, most_v = ref.attention(pool, q, lengths, policy, seg, tail, scale, max_rows)
    # A score is a sum of D exact products in fp32: off by D 2^-24 of the sum of their magnitudes at most.  A weight adds the
    # rounding of its argument, of exp2 and of the sums: 2^-20.  What the split weights lose: 2^-16 of a weight.
    delta = pool.D * 2.0 ** -24 * most_s + 2.0 ** -20
    half = 0.0 if out_fp32 else 2.0 ** -8 * (1 + 2.0 ** -7)
    err, bound = (out.double().cpu() - want).abs(), want.abs() * half + (2 * delta + 2.0 ** -16) * most_v
    assert (err <= bound).all(), f"out: {float((err - bound).max()):.3e} above the bound"
    empty = want_lse == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty)
    err = (lse.double().cpu() - want_lse)[~empty].abs()
    assert (err <= delta + 2.0 ** -22 * (1 + want_lse[~empty].abs())).all(), f"lse: {float(err.max()):.3e}"
    if accumulate:
        expected = before.clone()
        for (b, h), (rows, p) in weights.items():
            if policy[h] & 2:
                page, hh, r = pool.place(b, h, rows)
                expected[page, hh, r] += p
        got = pool.mass.double().cpu()
        assert torch.equal(got.isnan(), expected.isnan())
        added = (expected - before).nan_to_num()
        err = (got - expected).nan_to_num().abs()
        assert (err <= added * (4 * delta + 2.0 ** -20) + 2.0 ** -23 * expected.nan_to_num().abs() + 1e-30).all(), f"mass {float(err.max()):.3e}"
    return out, lse


KINDS = [dict(page_rows=16), dict(page_rows=32), dict(page_rows=1), dict(page_rows=7), dict(page_rows=96), dict(page_rows=64, per_head=True),
         dict(page_rows=20, per_head=True), dict(page_rows=64, token_major=True), dict(page_rows=64, e4m3=True),
         dict(page_rows=10, e4m3=True, per_head=True), dict(page_rows=32, e4m3=True, token_major=True)]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
@pytest.mark.parametrize("d,g", [(128, 4), (64, 1)])
def test_decode_of_ragged_lengths(kind, d, g):
    lengths = [0, 1, 31, 32, 33, 129, 517]
    pool = Pool(batch=7, hkv=2, d=d, max_pages=-(-520 // kind["page_rows"]), **kind).fill(lengths)
    _decode(pool, 2 * g, lengths)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 8, 16, 17, 40, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_of_any_group(g, d):
    lengths = [77, 300]
    pool = Pool(batch=2, hkv=1, d=d, page_rows=32, max_pages=10).fill(lengths)
    _decode(pool, g, lengths, accumulate=True)


@pytest.mark.parametrize("policy", [[0, 0, 0], [1, 1, 1], [0, 1, 2], [3, 2, 1]])
@pytest.mark.parametrize("page_rows,per_head", [(32, False), (16, True), (13, True)])
def test_decode_sees_what_the_policies_say(policy, page_rows, per_head):
    """Segments of 100 rows and a tail of 37, around a segment's start; pages before a window are gone."""
    lengths = [1, 100, 101, 137, 138, 250, 301]
    pool = Pool(batch=7, hkv=3, d=128, page_rows=page_rows, max_pages=-(-310 // page_rows), per_head=per_head).fill(lengths)
    if per_head:
        for b, n in enumerate(lengths):
            for h in range(3):
                pool.table[b, h, :ref.first_row(n, policy[h], 100, 37) // page_rows] = -7
    _decode(pool, 6, lengths, policy=policy, seg=100, tail=37)
    if 2 in policy:
        _decode(pool, 6, lengths, policy=policy, seg=100, tail=37, accumulate=True)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_of_many_windows_shares_the_rows_out(e4m3):
    """Over 64 windows a workgroup's slice goes on from one window into the next."""
    lengths = [(37 * i * i) % 700 for i in range(30)]
    pool = Pool(batch=30, hkv=4, d=64, page_rows=16, max_pages=44, e4m3=e4m3).fill(lengths)
    _decode(pool, 4, lengths, accumulate=True)
    _decode(pool, 4, lengths, out_fp32=False)


def test_decode_of_hundreds_of_windows():
    lengths = [1 + (i * 7919) % 65 for i in range(150)]
    pool = Pool(batch=150, hkv=2, d=64, page_rows=32, max_pages=3).fill(lengths)
    _decode(pool, 4, lengths, accumulate=True)


@pytest.mark.parametrize("batch,hkv", [(300, 1), (90, 6), (65, 1), (257, 1), (128, 2)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_decode_of_hundreds_of_windows_cut_evenly(batch, hkv, accumulate):
    """Room for rows that a workgroup would not take by itself, held by one sequence only: windows of every length, empty
    ones among them, shared out evenly; over 256 of them a thread of the search has more than one."""
    lengths = [[(7919 * (i + 3) * (h + 1)) % 130 * (i % 5 > 0) for h in range(hkv)] for i in range(batch)]
    lengths[batch // 2] = [1111] * hkv
    pool = Pool(batch=batch, hkv=hkv, d=128, page_rows=32, max_pages=35, spare=0)
    pool.fill(lengths)
    _decode(pool, 2 * hkv, lengths, accumulate=accumulate, policy=[2 + h % 2 for h in range(hkv)])


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
@pytest.mark.parametrize("d,g,batch", [(128, 4, 7), (64, 3, 7), (64, 1, 40)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_decode_of_ragged_lengths_in_a_roomy_table(kind, d, g, batch, accumulate):
    """The same lengths where the table has room for thousands of rows: windows are cut and joined."""
    lengths = [0, 1, 31, 32, 33, 129, 517]
    lengths = [lengths[i % 7] for i in range(batch)]
    pool = Pool(batch=batch, hkv=2, d=d, max_pages=-(-520 // kind["page_rows"]), **kind).fill(lengths)
    room = -(-4200 // kind["page_rows"])
    table = torch.full((*pool.table.shape[:-1], room), -1, dtype=torch.int32, device="cuda")
    table[..., :pool.max_pages] = pool.table
    pool.table, pool.max_pages = table, room
    _decode(pool, 2 * g, lengths, accumulate=accumulate)


@pytest.mark.parametrize("page_rows", [12, 32])
def test_weights_of_rows_that_lie_at_any_float(page_rows):
    lengths = [1, 3, 70, 1030]
    pool = Pool(batch=4, hkv=2, d=64, page_rows=page_rows, max_pages=-(-1100 // page_rows)).fill(lengths)
    for shift in (1, 2, 3):
        room = torch.full((pool.mass.numel() + 7,), 5.0, device="cuda")
        mass = room[shift:shift + pool.mass.numel()].view(pool.mass.shape)
        mass.copy_(pool.mass)
        pool.mass = mass
        _decode(pool, 4, lengths, accumulate=True)
        assert (room[:shift] == 5.0).all() and (room[shift + mass.numel():] == 5.0).all()


def test_counts_of_many_sequences():
    """More (sequence, head) pairs than a workgroup has threads, in and out of place."""
    B = 700
    pool = Pool(batch=B, hkv=3, d=64, page_rows=4, max_pages=1, mass=False, pos=False)
    pool.rows.copy_((torch.arange(B * 3, dtype=torch.int32, device="cuda") % 5).view(B, 3))
    m = [i % 4 for i in range(B)]
    cu = torch.tensor([sum(m[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    n = int(cu[-1])
    k = torch.ones((n, 3, 64), dtype=BF16, device="cuda")
    want = (pool.rows + torch.tensor(m, device="cuda")[:, None]).clamp(max=4).to(torch.int32)
    out = torch.empty_like(pool.rows)
    sa.seg_kv_paged_append(_cfg(pool, 3), pool.pages(), None, None, k, k, cu, n, 3, None, pool.rows, None, out, _stream())
    assert torch.equal(out, want)
    sa.seg_kv_paged_append(_cfg(pool, 3), pool.pages(), None, None, k, k, cu, n, 3, None, pool.rows, None, pool.rows, _stream())
    assert torch.equal(pool.rows, want)
    k = torch.ones((B, 3, 64), dtype=BF16, device="cuda")
    sa.seg_kv_paged_append(_cfg(pool, 3), pool.pages(), None, None, k, k, None, B, 1, None, pool.rows, None, pool.rows, _stream())
    assert torch.equal(pool.rows, (want + 1).clamp(max=4).to(torch.int32))


@pytest.mark.parametrize("batch,lengths", [(1, [40000]), (3, [9000, 70, 16385])])
@pytest.mark.parametrize("kind", [dict(page_rows=64), dict(page_rows=48, e4m3=True)], ids=["bf16", "e4m3"])
def test_decode_of_long_caches(batch, lengths, kind):
    pool = Pool(batch=batch, hkv=2, d=128, max_pages=-(-40960 // kind["page_rows"]), **kind).fill(lengths)
    _decode(pool, 8, lengths, accumulate=True)
    _decode(pool, 8, lengths, out_fp32=False, scale=0.3)


def test_decode_of_a_cache_with_holes_in_its_table():
    """Rows of pages that are not there are not seen, wherever they lie; a head without any has zeros."""
    for page_rows in (32, 24):
        pool = Pool(batch=4, hkv=2, d=64, page_rows=page_rows, max_pages=20).fill([450, 450, 450, 450])
        pool.table[0, 3], pool.table[0, 4], pool.table[0, 13] = -1, pool.n_pages, 2 ** 31 - 1
        pool.table[1, :] = -1
        pool.table[2, 1:] = -5
        _decode(pool, 8, [450] * 4, accumulate=True)


def test_decode_stops_at_the_rows_it_was_promised():
    pool = Pool(batch=2, hkv=2, d=64, page_rows=32, max_pages=20).fill([600, 33])
    _decode(pool, 4, [600, 33], max_rows=100, accumulate=True)
    pool.rows[0, 0] = -3  # nothing
    pool.rows[1, 1] = 2 ** 31 - 1  # as many as the table has, the rows behind 33 are NaN
    out, lse = torch.empty((2, 4, 64), dtype=BF16, device="cuda"), torch.empty((2, 4), device="cuda")
    cfg = _cfg(pool, 4)
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), 640)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    sa.seg_attn_decode_paged(cfg, pool.pages(), torch.ones((2, 4, 64), dtype=BF16, device="cuda"), pool.rows, 640, out, lse, ws, need, stream=_stream())
    assert (out[0, :2] == 0).all() and (lse[0, :2] == -math.inf).all() and out[0, 2:].isfinite().all() and out[1, 2:].isnan().all()


def test_decode_of_extreme_values():
    """Scores of both signs far apart, a row of infinities among the seen ones (NaN, as the formula), and none for others."""
    pool = Pool(batch=2, hkv=1, d=64, page_rows=16, max_pages=8).fill([100, 100])
    page, hh, r = pool.place(0, 0, [40])
    q = torch.ones((2, 2, 64), dtype=BF16, device="cuda")
    pool.k[page[0], 0, r[0]] = 200.0  # one row takes everything
    out, lse = _decode(pool, 2, [100, 100], q=q)
    assert torch.allclose(out[0, 0].cpu(), pool.v[page[0], 0, r[0]].float().cpu(), atol=1e-6)
    pool.k[page[0], 0, r[0]] = -3e38  # and one nothing
    _decode(pool, 2, [100, 100], q=q, scale=1e-3)
    pool.v[page[0], 0, r[0]] = float("inf")
    pool.k[page[0], 0, r[0]] = 0.0
    cfg = _cfg(pool, 2, out_fp32=True)
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), 128)
    ws, out, lse = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((2, 2, 64), device="cuda"), torch.empty((2, 2), device="cuda")
    sa.seg_attn_decode_paged(cfg, pool.pages(), q, pool.rows, 128, out, lse, ws, need, stream=_stream())
    assert not out[0].isfinite().any() and lse[0].isfinite().all() and out[1].isfinite().all()
    pool.k[page[0], 0, r[0]] = float("nan")
    sa.seg_attn_decode_paged(cfg, pool.pages(), q, pool.rows, 128, out, lse, ws, need, stream=_stream())
    assert out[0].isnan().all() and lse[0].isnan().all() and out[1].isfinite().all() and lse[1].isfinite().all()


def test_decode_agrees_with_the_arena_and_with_prefill():
    """The same tokens through seg_attn_fwd_seq (its last row) and through append and decode: segmented policies."""
    S, T, n, hq, policy = 96, 24, 331, 8, [0, 1, 2, 3]
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn((1, n, h, 128), generator=g).to(BF16).cuda() for h in (hq, 4, 4))
    pool = Pool(batch=1, hkv=4, d=128, page_rows=16, max_pages=30, mass=False, pos=False)
    cfg = _cfg(pool, hq, policy, S, T, out_fp32=True)
    out, lse = torch.empty((1, n, hq, 128), device="cuda"), torch.empty((1, hq, n), device="cuda")
    sa.seg_attn_fwd_seq(cfg, q, k, v, n, out, lse, _stream())
    sa.seg_kv_paged_append(cfg, pool.pages(), None, None, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n, None, pool.rows,
                           None, pool.rows, _stream())
    o, l = _decode(pool, hq, [n], policy=policy, seg=S, tail=T, q=q[:, -1].contiguous())
    # the prefill kernel rounds its weights to bf16 (2^-9 of each): the library's bar for it
    assert (o - out[:, -1]).abs().max() <= 1e-2 and (l - lse[:, :, -1]).abs().max() <= 1e-2


# ---- eviction --------------------------------------------------------------------------------------
def _evict(pool, keep, recent, first, policy=None, in_place=True, max_rows=None):
    policy = policy or [2] * pool.H
    want, moved = ref.evicted(pool, keep, recent, first, policy, max_rows)
    cfg = _cfg(pool, pool.H, policy)
    most = max_rows or pool.max_pages * pool.R
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pool.pages(), most, keep)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    rows_out = pool.rows if in_place else torch.full_like(pool.rows, -9)
    before = pool.rows.clone()
    sa.seg_kv_paged_evict(cfg, pool.pages(), pool.rows, most, keep, recent, first, rows_out, ws, need, _stream())
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(pool.rows, before)
        pool.rows = rows_out
    got = pool.state()
    for x in got:
        assert torch.equal(ref.bits(got[x]), ref.bits(want[x])), x
    return moved


@pytest.mark.parametrize("kind", [dict(page_rows=16), dict(page_rows=1), dict(page_rows=7, per_head=True), dict(page_rows=32, e4m3=True),
                                  dict(page_rows=24, e4m3=True, per_head=True), dict(page_rows=64, token_major=True)],
                         ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
@pytest.mark.parametrize("keep,recent,first", [(40, 10, 4), (1, 0, 0), (1, 1, 0), (64, 64, 0), (90, 0, 90), (200, 33, 5)])
@pytest.mark.parametrize("in_place", [True, False])
def test_eviction_matches_the_definition(kind, keep, recent, first, in_place):
    pool = Pool(batch=5, hkv=2, d=64, max_pages=-(-330 // kind["page_rows"]), **kind).fill([0, [40, 41], [64, 7], 201, [330, 129]])
    moved = _evict(pool, keep, recent, first, in_place=in_place)
    assert moved > 0 or recent + first >= keep or keep == 1
    pool.rows.clamp_(min=0)
    _evict(pool, max(1, keep // 2), recent // 2, first // 2)  # from rows that are out of order by now


def test_eviction_with_ties_zeros_and_what_is_no_weight():
    pool = Pool(batch=3, hkv=1, d=64, page_rows=16, max_pages=10).fill([150, 150, 150])
    page, hh, r = pool.place(0, 0, range(150))
    pool.mass[page.cuda(), 0, r.cuda()] = 0.25
    page, hh, r = pool.place(1, 0, range(150))
    odd = torch.tensor([0.0, -1.0, math.nan, -math.inf, math.inf, 1e-42, -0.0, 3.0]).repeat(19)[:150]
    pool.mass[page.cuda(), 0, r.cuda()] = odd.cuda()
    page, hh, r = pool.place(2, 0, range(150))
    pool.mass[page.cuda(), 0, r.cuda()] = (torch.arange(150) % 3).float().cuda()
    _evict(pool, 61, 8, 2)


def test_eviction_leaves_heads_without_the_past_alone():
    pool = Pool(batch=2, hkv=4, d=64, page_rows=16, max_pages=10, per_head=True).fill([150, 100])
    _evict(pool, 50, 5, 1, policy=[1, 2, 0, 3])
    assert pool.rows.tolist() == [[150, 50, 150, 50], [100, 50, 100, 50]]


@pytest.mark.parametrize("n,keep", [(1023, 512), (1025, 1024), (5000, 200), (40001, 20000), (70001, 69990), (40001, 50000), (80003, 40000)])
def test_eviction_of_long_heads(n, keep):
    pool = Pool(batch=1, hkv=2, d=64, page_rows=64, max_pages=-(-n // 64)).fill([[n, n - 13]])
    _evict(pool, keep, keep // 10, 4)


def test_eviction_of_a_table_with_holes_and_of_a_promise():
    pool = Pool(batch=2, hkv=1, d=64, page_rows=16, max_pages=10).fill([150, 150])
    pool.table[0, 2], pool.table[0, 8] = -1, pool.n_pages
    _evict(pool, 60, 8, 2)
    pool = Pool(batch=2, hkv=1, d=64, page_rows=16, max_pages=10).fill([150, 90])
    _evict(pool, 60, 8, 2, max_rows=100)
    pool = Pool(batch=2, hkv=1, d=64, page_rows=16, max_pages=10).fill([150, 90])
    _evict(pool, 160, 8, 2)  # nobody holds as much
    _evict(pool, 10 ** 12, 10 ** 11, 2)


def test_pools_beyond_32_bits_of_offset():
    """600,000 pages of 16 KB: the same sequences in a small pool and in a large one, through append, decode and eviction."""
    small, large = (Pool(batch=2, hkv=2, d=128, page_rows=64, max_pages=12, per_head=True, spare=n, seed=n).fill([500, 700]) for n in (0, 600000))
    assert int(large.table.max()) * large.k.stride(0) * 2 > 2 ** 32
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((2, h, 128), generator=g).to(BF16).cuda() for h in (8, 2, 2))
    for pool in (small, large):
        sa.seg_kv_paged_append(_cfg(pool, 8), pool.pages(), None, None, k, v, None, 2, 1, torch.tensor([500, 700], device="cuda"), pool.rows, None,
                               pool.rows, _stream())
        _decode(pool, 8, [501, 701], q=q, accumulate=True)
    cfg = _cfg(small, 2)
    for pool in (small, large):
        need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pool.pages(), 768, 300)
        sa.seg_kv_paged_evict(cfg, pool.pages(), pool.rows, 768, 300, 30, 4, pool.rows, torch.empty(need, dtype=torch.uint8, device="cuda"), need, _stream())
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(2):
            for x, y in zip(small.kv(b, h, range(300)), large.kv(b, h, range(300))):
                assert torch.equal(x, y)
            for name in ("mass", "pos"):
                x, y = (getattr(p, name)[p.place(b, h, range(300))[0].cuda(), 0, (torch.arange(300) % 64).cuda()] for p in (small, large))
                assert torch.equal(x, y), name


# ---- together --------------------------------------------------------------------------------------
def test_prompt_then_steps_that_accumulate_then_evict():
    """A program's loop: prompt appended turned, steps of append and decode that add up weights, an eviction every
    fourth step; after every step the attention is what the definition gives for the rows that are held."""
    B, hq, hkv, d, rope = 3, 8, 2, 64, dict(theta=10000.0)
    g = torch.Generator().manual_seed(12)
    for e4m3 in (False, True):
        pool = Pool(batch=B, hkv=hkv, d=d, page_rows=16, max_pages=14, e4m3=e4m3)
        cfg, r = _cfg(pool, hq), sa.make_rope(**rope)
        m = [150, 31, 97]
        cu = torch.tensor([0, 150, 181, 278], dtype=torch.int32, device="cuda")
        k, v = (torch.randn((278, hkv, d), generator=g).to(BF16).cuda() for _ in "kv")
        q = torch.randn((278, hq, d), generator=g).to(BF16).cuda()
        sa.seg_kv_paged_append(cfg, pool.pages(), r, q, k, v, cu, 278, 150, None, pool.rows, q, pool.rows, _stream())
        at = torch.tensor(m, dtype=torch.int64, device="cuda")
        for step in range(9):
            k, v = (torch.randn((B, hkv, d), generator=g).to(BF16).cuda() for _ in "kv")
            q = torch.randn((B, hq, d), generator=g).to(BF16).cuda()
            sa.seg_kv_paged_append(cfg, pool.pages(), r, q, k, v, None, B, 1, at, pool.rows, q, pool.rows, _stream())
            at += 1
            _decode(pool, hq, pool.rows.tolist(), accumulate=True, q=q)
            if step % 4 == 3:
                _evict(pool, 64, 16, 2)
        assert int(pool.pos.max()) == 158


def test_captured_steps_replay_while_the_cache_grows():
    """Append, decode with weights and eviction in one graph, replayed between eager work; every replay against eager calls
    on a copy of the pool, bit by bit (the kernels add in a fixed order)."""
    B, hq, hkv, d = 2, 8, 2, 128
    pools = [Pool(batch=B, hkv=hkv, d=d, page_rows=32, max_pages=12).fill([100, 240]) for _ in range(2)]
    cfg, rope = _cfg(pools[0], hq), sa.make_rope(theta=10000.0)
    most = 12 * 32
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pools[0].pages(), most, True)
    need_e = sa.seg_kv_paged_evict_workspace_bytes(cfg, pools[0].pages(), most, 250)
    static = [dict(q=torch.empty((B, hq, d), dtype=BF16, device="cuda"), qo=torch.empty((B, hq, d), dtype=BF16, device="cuda"),
                   k=torch.empty((B, hkv, d), dtype=BF16, device="cuda"), v=torch.empty((B, hkv, d), dtype=BF16, device="cuda"),
                   at=torch.tensor([100, 240], device="cuda"), out=torch.empty((B, hq, d), dtype=BF16, device="cuda"),
                   lse=torch.empty((B, hq), device="cuda"), ws=torch.empty(need, dtype=torch.uint8, device="cuda"),
                   we=torch.empty(need_e, dtype=torch.uint8, device="cuda"), pages=p.pages()) for p in pools]

    def step(i):
        s, p = static[i], pools[i]
        sa.seg_kv_paged_append(cfg, s["pages"], rope, s["q"], s["k"], s["v"], None, B, 1, s["at"], p.rows, s["qo"], p.rows, _stream())
        sa.seg_attn_decode_paged(cfg, s["pages"], s["qo"], p.rows, most, s["out"], s["lse"], s["ws"], need, accumulate=True, stream=_stream())
        sa.seg_kv_paged_evict(cfg, s["pages"], p.rows, most, 250, 20, 4, p.rows, s["we"], need_e, _stream())

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(0)
    g = torch.Generator().manual_seed(2)
    for i in range(20):
        for x, h in (("q", hq), ("k", hkv), ("v", hkv)):
            new = torch.randn((B, h, d), generator=g).to(BF16).cuda()
            static[0][x].copy_(new)
            static[1][x].copy_(new)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        for a, b in ((pools[0].state(), pools[1].state()), (static[0], static[1])):
            for x in a:
                if x not in ("ws", "we", "pages"):
                    assert torch.equal(ref.bits(a[x]), ref.bits(b[x])), (i, x)
        for s in static:
            s["at"] += 1
    assert pools[0].rows.tolist() == [[120] * 2, [250] * 2]


def test_two_streams_with_a_workspace_each():
    pools = [Pool(batch=1, hkv=2, d=128, page_rows=64, max_pages=300, seed=i).fill([19000 - i], seed=i + 5) for i in range(2)]
    cfg = _cfg(pools[0], 8, out_fp32=True)
    q = torch.randn((1, 8, 128), generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pools[0].pages(), 19000)

    def call(p, stream):
        ws, out, lse = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((1, 8, 128), device="cuda"), torch.empty((1, 8), device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        sa.seg_attn_decode_paged(cfg, p.pages(), q, p.rows, 19000, out, lse, ws, need, stream=stream.cuda_stream)
        return out, lse, ws

    alone = []
    for p in pools:
        alone.append(call(p, torch.cuda.current_stream()))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pools]
    both = [call(p, s) for _ in range(5) for p, s in zip(pools, streams)]
    torch.cuda.synchronize()
    for i, x in enumerate(both):
        assert torch.equal(x[0], alone[i % 2][0]) and torch.equal(x[1], alone[i % 2][1])
