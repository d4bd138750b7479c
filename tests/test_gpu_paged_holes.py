"""Eviction from caches whose tables have holes: what has to be there afterwards, by the rows' positions and without
a word about which row moves where."""
import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref
from paged_ref import Pool

pytestmark = pytest.mark.gpu


def _held(pool, b, h, n):
    """{position: (contents, row)} of the rows below n that have a page."""
    page, hh, r = pool.place(b, h, range(n))
    rows = torch.arange(n)[page >= 0]
    at = page[rows].cuda(), hh, r[rows].cuda()
    x = [ref.bits(y[at]) for y in (pool.k, pool.v)] + [ref.bits(pool.mass[at])[:, None]]
    if pool.e4m3:
        x += [y[at].cpu()[:, None] for y in (pool.k_scale, pool.v_scale)]
    x = torch.cat([y.to(torch.int64) for y in x], 1)
    return {p: (x[i], int(rows[i])) for i, p in enumerate(pool.pos[at].tolist())}


def _stays(before, keep, recent, first, mass):
    """Positions that have to stay: as many as rows below keep are there, newest and first ones first, then the heaviest
    (all weights differ)."""
    newest = max(before)
    order = sorted(before, key=lambda p: (p > newest - recent, p if p > newest - recent else 0, p < first, 0 if p < first else mass[p]), reverse=True)
    return set(order[:sum(i < keep for _, i in before.values())])


def _evict(pool, keep, recent, first, most=None):
    cfg = sa.make_config(batch=pool.B, n_q_heads=pool.H, n_kv_heads=pool.H, head_dim=pool.D, seg_len=64, tail_len=16, kv_policy=[2] * pool.H)
    most = most or pool.max_pages * pool.R
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pool.pages(), most, keep)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_evict(cfg, pool.pages(), pool.rows, most, keep, recent, first, pool.rows, ws, need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("page_rows,n,keep,recent,first,holes", [
    (16, 70, 64, 8, 0, [3]),                  # the newest rows are among those that have to move
    (16, 150, 60, 8, 2, [2, 8]),
    (16, 150, 60, 8, 2, [0]),                 # the first rows are not there
    (16, 160, 40, 30, 0, [0, 1]),             # fewer places than newest rows
    (16, 160, 40, 20, 4, [0, 2, 9]),          # row keep inside a hole; the newest row is not there
    (16, 160, 48, 8, 0, [0, 1, 2]),           # no place at all below row keep
    (1, 90, 40, 10, 3, [0, 5, 6, 39, 40, 77]),
    (64, 5000, 4500, 300, 4, [0, 33, 69, 70, 75]),
    (64, 5000, 300, 50, 4, [1, 5, 77]),
    (24, 5000, 4500, 300, 4, [0, 33, 69, 187, 188]),
    (192, 9000, 2000, 300, 4, [3, 10, 20, 46]),
])
@pytest.mark.parametrize("e4m3", [False, True])
def test_what_has_to_stay_stays_where_the_table_has_holes(page_rows, n, keep, recent, first, holes, e4m3):
    pool = Pool(batch=2, hkv=1, d=64, page_rows=page_rows, max_pages=-(-n // page_rows), e4m3=e4m3).fill([n, n - 3])
    pool.table[0, torch.tensor(holes)] = -1
    pool.table[1, holes[0]] = pool.n_pages
    pool.mass.copy_(torch.randperm(pool.mass.numel(), generator=torch.Generator().manual_seed(6)).view(pool.mass.shape) / 1000)
    before = [_held(pool, b, 0, m) for b, m in enumerate((n, n - 3))]
    stays = []
    for b in range(2):
        mass = {p: float(x[0][2 * pool.D].to(torch.int32).view(torch.float32)) for p, x in before[b].items()}
        assert len(set(mass.values())) == len(mass)
        stays.append(_stays(before[b], keep, recent, first, mass))
    _evict(pool, keep, recent, first)
    assert pool.rows.tolist() == [[keep]] * 2
    for b in range(2):
        got = _held(pool, b, 0, keep)
        assert set(got) == stays[b], f"sequence {b}: missing {sorted(stays[b] - set(got))[:9]}, there {sorted(set(got) - stays[b])[:9]}"
        for p, (x, row) in got.items():
            assert torch.equal(x, before[b][p][0]), p
            assert row == before[b][p][1] or before[b][p][1] >= keep, p  # rows below keep do not change places


def test_nothing_moves_where_nothing_is_there():
    pool = Pool(batch=3, hkv=2, d=64, page_rows=16, max_pages=10).fill([150, 150, 150])
    pool.table[0, :] = -1
    pool.table[1, :4] = -1
    before = pool.state()
    _evict(pool, 60, 8, 2)
    assert pool.rows.tolist() == [[60] * 2] * 3
    other = pool.table[2].long()
    for x in ("k", "v", "mass", "pos"):
        a, b = before[x].clone(), getattr(pool, x).clone()
        a[other], b[other] = 0, 0
        assert torch.equal(ref.bits(a), ref.bits(b)), x
