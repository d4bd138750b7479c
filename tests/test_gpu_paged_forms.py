"""Forms of the paged operators that only large calls take: several tokens per workgroup of an append, many steps per wave of an
eviction in pages of every kind, keys in the workspace; and a row that is seen but weighs nothing."""
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


def _cfg(batch, hq, hkv, d, **kw):
    return sa.make_config(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seg_len=64, tail_len=16, kv_policy=[2] * hkv, **kw)


# ---- append ----------------------------------------------------------------------------------------
ROPES = [dict(theta=10000.0), dict(theta=10000.0, interleaved=True, magnitude=1.25), dict(theta=10000.0, rotary_dim=32, interleaved=True),
         dict(theta=10000.0, rotary_dim=48)]


def _near(got, exact, size):
    """bf16: half a step (2^-8) of the value, and the turning's own 2^-20 of the magnitudes that meet in it."""
    return ((got.double().cpu() - exact).abs() <= exact.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + size * 2.0 ** -20).all()


def _check_tokens(pool, b, row, position, q, k, v, q_out, rope):
    """Token t is row[t, h] of sequence b[t]: what append has to have written for it."""
    T, H = k.shape[:2]
    exact, size = ref.turned(k.double().cpu(), position, rope)
    page, at = [], []
    for h in range(H):
        table = (pool.table[:, h] if pool.per_head else pool.table).cpu().long()
        page.append(table[b, row[:, h] // pool.R])
        at.append(row[:, h] % pool.R)
    page, at = torch.stack(page, 1), torch.stack(at, 1)
    head = torch.zeros(T, H, dtype=torch.int64) if pool.per_head else torch.arange(H).expand(T, H)
    place = page.cuda(), head.cuda(), at.cuda()
    assert torch.equal(pool.pos[place].cpu(), position.to(torch.int32)[:, None].expand(T, H))
    assert not pool.mass[place].any()
    if pool.e4m3:
        bits, scale = ref.e4m3_rows(v.double().cpu().flatten(0, 1))
        assert torch.equal(pool.v[place].cpu().flatten(0, 1), bits) and torch.equal(pool.v_scale[place].cpu().flatten(), scale)
        s = torch.exp2(pool.k_scale[place].double().cpu() - 127)
        most = exact.abs().amax(-1)
        assert (most * (1 - 2.0 ** -18) <= 448 * s).all() and (most * (1 + 2.0 ** -18) > 224 * s).all()
        err = (pool.k[place].cpu().view(torch.float8_e4m3fn).double() * s[..., None] - exact).abs()
        # half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below 2^-6), and the turning's own error
        assert (err <= exact.abs() * 2.0 ** -4 + 2.0 ** -10 * s[..., None] + size * 2.0 ** -19).all()
    else:
        assert torch.equal(pool.v[place].cpu(), v.cpu()) and _near(pool.k[place], exact, size)
    assert _near(q_out, *ref.turned(q.double().cpu(), position, rope))


@pytest.mark.parametrize("total", [2049, 3301, 4399, 8005])
@pytest.mark.parametrize("rope", ROPES, ids=lambda r: "-".join(f"{a}{b}" for a, b in r.items()))
@pytest.mark.parametrize("e4m3,d,per_head", [(False, 64, False), (True, 128, True)])
def test_append_of_prompts_that_end_inside_a_workgroup(total, rope, e4m3, d, per_head):
    """Sequences of 0 to 12 tokens and a long one; a workgroup has two to four tokens."""
    hq, hkv, new = 4, 2, []
    while sum(new) + 700 < total:
        new.append((5 * len(new) * len(new) + 3) % 13)
    new.insert(len(new) // 2, total - sum(new))
    B, longest = len(new), max(new)
    pool = Pool(batch=B, hkv=hkv, d=d, page_rows=24, max_pages=-(-(longest + 40) // 24), e4m3=e4m3, per_head=per_head, spare=0)
    held = (torch.arange(B * hkv).view(B, hkv) * 7) % 31
    pool.rows.copy_(held)
    g = torch.Generator().manual_seed(total)
    q, k, v = (torch.randn((total, h, d), generator=g).to(BF16).cuda() for h in (hq, hkv, hkv))
    cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    pos0 = torch.randint(0, 100000, (B,), generator=g, dtype=torch.int64)
    q_out = torch.empty_like(q)
    sa.seg_kv_paged_append(_cfg(B, hq, hkv, d), pool.pages(), sa.make_rope(**rope), q, k, v, cu.cuda(), total, longest, pos0.cuda(), pool.rows, q_out,
                           pool.rows, _stream())
    assert torch.equal(pool.rows.cpu().long(), held + torch.tensor(new)[:, None])
    b = torch.repeat_interleave(torch.arange(B), torch.tensor(new))
    i = torch.arange(total) - cu[b].long()
    _check_tokens(pool, b, held[b] + i[:, None], pos0[b] + i, q, k, v, q_out, rope)


@pytest.mark.parametrize("batch", [2048, 4500])
@pytest.mark.parametrize("rope", ROPES[:2], ids=["half", "interleaved"])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_a_token_each_for_thousands(batch, rope, e4m3, in_place):
    hq, hkv, d = 2, 1, 64
    pool = Pool(batch=batch, hkv=hkv, d=d, page_rows=8, max_pages=2, e4m3=e4m3, spare=0)
    held = (torch.arange(batch)[:, None] * 5) % 16
    pool.rows.copy_(held)
    g = torch.Generator().manual_seed(batch)
    q, k, v = (torch.randn((batch, h, d), generator=g).to(BF16).cuda() for h in (hq, hkv, hkv))
    pos0 = torch.randint(0, 100000, (batch,), generator=g, dtype=torch.int64)
    q_out, out = torch.empty_like(q), pool.rows if in_place else torch.full_like(pool.rows, -1)
    sa.seg_kv_paged_append(_cfg(batch, hq, hkv, d), pool.pages(), sa.make_rope(**rope), q, k, v, None, batch, 1, pos0.cuda(), pool.rows, q_out, out, _stream())
    assert torch.equal(out.cpu().long(), held + 1)
    _check_tokens(pool, torch.arange(batch), held, pos0, q, k, v, q_out, rope)


# ---- eviction --------------------------------------------------------------------------------------
@pytest.mark.parametrize("page_rows,per_head,e4m3", [(16, False, False), (24, True, False), (1, False, False), (64, True, True), (192, False, False)])
@pytest.mark.parametrize("n,keep,levels", [(4096, 1000, 0), (4097, 4000, 5), (5000, 2000, 0), (32768, 30000, 0), (32769, 32000, 9), (40003, 20000, 0)])
def test_eviction_of_many_rows_in_any_pages(page_rows, per_head, e4m3, n, keep, levels):
    """Both sides of 4096 rows (a wave has more than four steps, table entries are asked for again) and of 32768 (keys in the
    workspace); `levels`: so few different weights that most of them are equal."""
    pool = Pool(batch=1, hkv=2, d=64, page_rows=page_rows, max_pages=-(-n // page_rows), per_head=per_head, e4m3=e4m3, spare=0).fill([[n, n - 5]])
    if levels:
        pool.mass.copy_((pool.mass.nan_to_num() * levels).floor())
    want, moved = ref.evicted(pool, keep, keep // 7, 4, [2, 2])
    assert moved > 0
    cfg, most = _cfg(1, 2, 2, 64), pool.max_pages * page_rows
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pool.pages(), most, keep)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_evict(cfg, pool.pages(), pool.rows, most, keep, keep // 7, 4, pool.rows, ws, need, _stream())
    got = pool.state()
    for x in got:
        assert torch.equal(ref.bits(got[x]), ref.bits(want[x])), x


# ---- decode ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("room", [128, 16384], ids=["whole", "cut"])
def test_decode_past_a_row_that_weighs_nothing(room):
    """One row's score is some 10^34 below the others': out and lse are those of the other rows, to the ordinary tolerance (a
    score is off by D 2^-24 of its products' magnitudes, a weight by 2^-20 more)."""
    pool = Pool(batch=2, hkv=1, d=64, page_rows=16, max_pages=8, mass=False).fill([100, 100])
    (page,), _, (r,) = pool.place(0, 0, [40])
    pool.k[page, 0, r] = -3e38
    table = torch.full((2, room // 16), -1, dtype=torch.int32, device="cuda")
    table[:, :8] = pool.table
    pool.table, pool.max_pages = table, room // 16
    q = torch.ones((2, 2, 64), dtype=BF16, device="cuda")
    scale = 1e-3
    cfg = _cfg(2, 2, 1, 64, scale=scale, out_fp32=True)
    out, lse = torch.empty((2, 2, 64), device="cuda"), torch.empty((2, 2), device="cuda")
    need = sa.seg_attn_decode_paged_workspace_bytes(cfg, pool.pages(), room)
    sa.seg_attn_decode_paged(cfg, pool.pages(), q, pool.rows, room, out, lse, torch.empty(need, dtype=torch.uint8, device="cuda"), need, stream=_stream())
    for b in range(2):
        rows = [i for i in range(100) if b == 1 or i != 40]
        k, v = pool.kv(b, 0, rows)
        s = k.sum(-1) * scale
        delta = 64 * 2.0 ** -24 * float(k.abs().sum(-1).max()) * scale + 2.0 ** -20
        want_lse = float(torch.logsumexp(s, 0))
        want = (s - want_lse).exp() @ v
        for h in range(2):
            assert abs(float(lse[b, h]) - want_lse) <= delta + 2.0 ** -22 * (1 + abs(want_lse)), (b, h)
            assert ((out[b, h].double().cpu() - want).abs() <= (2 * delta + 2.0 ** -16) * float(v.abs().max())).all(), (b, h)
        assert math.isfinite(want_lse)
