"""Sparse attention over a paged cache and the tables under it, against their definitions (sparse_ref.py)."""
import math

import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref
import sparse_ref as sref
from paged_ref import Pool

pytestmark = pytest.mark.gpu
BF16, I32, I64 = torch.bfloat16, torch.int32, torch.int64


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _cfg(pool, hq, policy=None, seg=64, tail=16, **kw):
    return sa.make_config(batch=pool.B, n_q_heads=hq, n_kv_heads=pool.H, head_dim=pool.D, seg_len=seg, tail_len=tail,
                          kv_policy=policy or [2] * pool.H, **kw)


def _sums(new):
    return [sum(new[:i]) for i in range(len(new) + 1)]


# ---- tables ----------------------------------------------------------------------------------------
class Tables:
    """A table without memory behind it: pages in any order for rows that are held."""

    def __init__(self, *, rows, page_rows, max_pages, per_head=False, policy, seg=64, tail=16, n_pages, seed=0, windows_only=False):
        self.B, self.H, self.D, self.rows, self.R, self.max_pages, self.per_head = len(rows), len(rows[0]), 64, rows, page_rows, max_pages, per_head
        self.policy, self.seg, self.tail, self.n_pages = policy, seg, tail, n_pages
        g = torch.Generator().manual_seed(seed)
        pages = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((self.B, self.H, max_pages) if per_head else (self.B, max_pages), -1, dtype=I32)
        self.users = torch.zeros(n_pages, dtype=I32)
        for b in range(self.B):
            for h in range(self.H if per_head else 1):
                held = set()
                for k in ([h] if per_head else range(self.H)):
                    lo = ref.first_row(rows[b][k], policy[k], seg, tail) if windows_only else 0
                    held |= {r // page_rows for r in range(lo, min(rows[b][k], max_pages * page_rows))}
                for e in held:
                    page = pages.pop()
                    self.users[page] = 1
                    (self.table[b, h] if per_head else self.table[b])[e] = page

    def take_away(self, left, seed=1):
        """All but `left` of the free pages belong to somebody else."""
        free = (self.users <= 0).nonzero()[:, 0]
        self.users[free[torch.randperm(len(free), generator=torch.Generator().manual_seed(seed))[left:]]] = 1

    def device(self):
        self.t, self.u = self.table.cuda(), self.users.cuda()
        self.dummy = torch.empty(256, dtype=torch.uint8, device="cuda")  # no call here reads keys or values
        return sa.make_pages(k=self.dummy, v=self.dummy, table=self.t, max_pages=self.max_pages, page_rows=self.R, n_pages=self.n_pages,
                             per_head=self.per_head)

    def common(self):
        return dict(table=self.table, users=self.users, rows=self.rows, page_rows=self.R, per_head=self.per_head, policy=self.policy,
                    seg=self.seg, tail=self.tail)

    def reserve(self, new, newest=False, slots=True, total=None, cu="given"):
        pages, cfg = self.device(), _cfg(self, self.H, self.policy, self.seg, self.tail)
        sums = _sums(new)
        total = total or max(1, sums[-1])
        granted = torch.full((self.B,), -9, dtype=I32, device="cuda")
        at = torch.full((total, self.H), -9, dtype=I64, device="cuda") if slots else None
        need = sa.seg_kv_paged_reserve_workspace_bytes(cfg, pages)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        rows = torch.tensor(self.rows, dtype=I32, device="cuda")
        sa.seg_kv_paged_reserve(cfg, pages, self.u, torch.tensor(sums, dtype=I32, device="cuda") if cu else None, total, max(1, max(new)), rows,
                                granted, at, ws, need, newest_only=newest, stream=_stream())
        want = sref.reserved(new=new, newest=newest, slots=torch.full((total, self.H), -9, dtype=I64) if slots else None, cu=sums, **self.common())
        assert self.t.cpu().tolist() == want[0].tolist()
        assert self.u.cpu().tolist() == want[1].tolist()
        assert granted.tolist() == want[2]
        if slots:
            assert at.cpu().tolist() == want[3].tolist()
        return want


P3 = [3, 1, 0]
RESERVES = [
    dict(rows=[[5, 9, 0], [0, 0, 0], [64, 64, 64]], page_rows=16, new=[30, 0, 1]),
    dict(rows=[[5, 9, 0], [0, 0, 0], [64, 64, 64]], page_rows=16, per_head=True, new=[30, 7, 100]),
    dict(rows=[[100, 300, 300], [300, 100, 170]], page_rows=8, new=[90, 11]),
    dict(rows=[[100, 300, 300], [300, 100, 170]], page_rows=8, per_head=True, new=[90, 11]),
    dict(rows=[[3, 3, 3]] * 7, page_rows=1, new=[1, 2, 0, 5, 1, 1, 40]),
    dict(rows=[[0, 0, 0]] * 4, page_rows=24, per_head=True, new=[200, 1, 65, 64]),
]


@pytest.mark.parametrize("newest", [False, True], ids=["all", "newest"])
@pytest.mark.parametrize("left", [None, 9, 0], ids=["enough", "nine", "none"])
@pytest.mark.parametrize("kind", RESERVES, ids=range(len(RESERVES)))
def test_reserve(kind, left, newest):
    kind = dict(kind)
    new = kind.pop("new")
    t = Tables(max_pages=420 // kind["page_rows"] + 1, policy=P3, n_pages=2000, windows_only=newest, **kind)
    if left is not None:
        t.take_away(left)
    t.reserve(new, newest)


def test_reserve_of_one_token_each_without_cu_seqlens():
    rows = [[i * 16 + (i % 3), i * 16, 33] for i in range(60)]
    Tables(rows=rows, page_rows=16, max_pages=70, policy=P3, n_pages=9000).reserve([1] * 60, cu=None)
    Tables(rows=rows, page_rows=16, max_pages=70, policy=P3, n_pages=9000, per_head=True).reserve([1] * 60, cu=None, slots=False)


def test_reserve_of_sequences_that_do_not_fit_their_table():
    t = Tables(rows=[[60, 64, 2], [10, 10, 10], [70, 70, 70], [0, 0, 0]], page_rows=8, max_pages=8, policy=P3, n_pages=100)
    want = t.reserve([1, 54, 1, 65])
    assert want[2] == [0, 1, 0, 0]


def test_reserve_leaves_tokens_behind_the_last_sequence_and_finds_reserved_pages():
    t = Tables(rows=[[5, 5, 5], [0, 0, 0]], page_rows=8, max_pages=20, policy=P3, n_pages=60)
    want = t.reserve([20, 3], total=40)
    t.table, t.users = want[0], want[1]
    again = t.reserve([20, 3], total=40)  # all there already
    assert again[0].tolist() == want[0].tolist() and again[2] == [1, 1]


@pytest.mark.parametrize("n_pages", [40, 1 << 19])
def test_reserve_for_a_batch_without_tokens_grants_and_changes_nothing(n_pages):
    """Either way of reserving: by one workgroup, and by launches for many pages."""
    t = Tables(rows=[[5, 9, 0], [200, 0, 0]], page_rows=16, max_pages=16, policy=P3, n_pages=n_pages)
    pages, cfg = t.device(), _cfg(t, t.H, P3)
    granted = torch.full((2,), -9, dtype=I32, device="cuda")
    need = sa.seg_kv_paged_reserve_workspace_bytes(cfg, pages)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_reserve(cfg, pages, t.u, torch.zeros(3, dtype=I32, device="cuda"), 0, 1, torch.tensor(t.rows, dtype=I32, device="cuda"), granted,
                            torch.empty((0, 3), dtype=I64, device="cuda"), ws, need, stream=_stream())
    assert granted.tolist() == [1, 1]
    assert torch.equal(t.u.cpu(), t.users) and torch.equal(t.t.cpu(), t.table)


def test_reserve_over_many_chunks_of_pages():
    t = Tables(rows=[[0, 0, 0]] * 9, page_rows=4, max_pages=1400, policy=[2, 2, 2], n_pages=40000, per_head=True)
    t.users[torch.rand(40000, generator=torch.Generator().manual_seed(3)) < 0.7] = 1
    t.users[::7] = 2
    t.users[5::1000] = -3  # free as well
    t.reserve([5000, 3, 1, 999, 0, 5000, 17, 1, 400])


RELEASES = [
    dict(rows=[[200, 200, 200], [0, 0, 0], [65, 64, 63], [1, 130, 400]], page_rows=16),
    dict(rows=[[200, 200, 200], [0, 0, 0], [65, 64, 63], [1, 130, 400]], page_rows=16, per_head=True),
    dict(rows=[[399, 128, 129]], page_rows=1), dict(rows=[[399, 128, 129]], page_rows=5, per_head=True),
]


@pytest.mark.parametrize("kind", RELEASES, ids=range(len(RELEASES)))
@pytest.mark.parametrize("policy", [P3, [1, 1, 1], [0, 0, 2]])
def test_release(kind, policy):
    t = Tables(max_pages=420 // kind["page_rows"] + 1, policy=policy, n_pages=2000, **kind)
    t.users[::3] += 1  # named by other tables too
    full = t.table.clone()
    t.rows = [[max(0, n - 37) for n in r] for r in t.rows]
    t.table.view(-1)[::11] = t.n_pages + 5  # names nothing: left alone
    pages = t.device()
    sa.seg_kv_paged_release(_cfg(t, t.H, policy, t.seg, t.tail), pages, t.u, torch.tensor(t.rows, dtype=I32, device="cuda"), stream=_stream())
    table, users = sref.released(**t.common())
    assert t.t.cpu().tolist() == table.tolist() and t.u.cpu().tolist() == users.tolist()
    assert table.tolist() != full.tolist()


def test_release_of_a_page_that_several_entries_name():
    t = Tables(rows=[[40, 40, 40]] * 5, page_rows=8, max_pages=5, policy=[2, 2, 2], n_pages=40)
    t.table[1:] = t.table[0]
    t.users[:] = 0
    t.users[t.table[0].long()] = 5
    t.rows = [[0, 0, 0], [17, 17, 17], [0, 0, 0], [40, 40, 40], [0, 0, 0]]
    pages = t.device()
    sa.seg_kv_paged_release(_cfg(t, 3, [2, 2, 2]), pages, t.u, torch.tensor(t.rows, dtype=I32, device="cuda"), stream=_stream())
    table, users = sref.released(**t.common())
    assert t.t.cpu().tolist() == table.tolist() and t.u.cpu().tolist() == users.tolist()


# ---- bounds ----------------------------------------------------------------------------------------
BLOCKS = [dict(page_rows=16, block=16), dict(page_rows=64, block=64, per_head=True), dict(page_rows=96, block=48), dict(page_rows=64, block=32, token_major=True),
          dict(page_rows=32, block=32, e4m3=True), dict(page_rows=128, block=64, e4m3=True, per_head=True), dict(page_rows=48, block=16, e4m3=True, token_major=True)]


def _name(k):
    return "-".join(f"{a}{b}" for a, b in k.items())


def _pool(kind, lengths, *, d=128, hkv=2, seed=0, **kw):
    kind = dict(kind)
    block = kind.pop("block")
    most = max(max(x) if isinstance(x, list) else x for x in lengths)
    pool = Pool(batch=len(lengths), hkv=hkv, d=d, max_pages=-(-(most + 1) // kind["page_rows"]), **kind, seed=seed, **kw).fill(lengths, seed=seed + 1)
    return pool, sref.Blocks(pool, block)


def _list(pool):
    return pool.rows.cpu().tolist()


def _summarize(pool, blocks, rows_from, max_new, policy):
    rows = _list(pool)
    want = sref.summarized(pool, blocks, rows_from or [[0] * pool.H] * pool.B, rows, policy, max_new)
    sa.seg_kv_paged_summarize(_cfg(pool, pool.H, policy), pool.pages(), blocks.c,
                              torch.tensor(rows_from, dtype=I32, device="cuda") if rows_from else None, pool.rows, max_new, stream=_stream())
    assert torch.equal(blocks.bounds.cpu(), want[0]) and torch.equal(blocks.scale.cpu(), want[1])


@pytest.mark.parametrize("kind", BLOCKS, ids=_name)
@pytest.mark.parametrize("d", [64, 128])
def test_summarize(kind, d):
    lengths = [0, 1, 15, [16, 300], [200, 64], 130]
    pool, blocks = _pool(kind, lengths, d=d)
    _summarize(pool, blocks, None, 301, [2, 3])
    pool, blocks = _pool(kind, lengths, d=d, seed=5)
    _summarize(pool, blocks, [[0, 0], [0, 0], [3, 15], [15, 100], [199, 63], [131, 7]], 60, [2, 3])
    pool, blocks = _pool(kind, lengths, d=d, seed=6)
    _summarize(pool, blocks, None, 300, [1, 2])


def test_summarize_of_every_magnitude():
    """Zeros, one large element, tiny ones, borders of the scale, infinities and NaN."""
    for e4m3 in (False, True):
        pool, blocks = _pool(dict(page_rows=16, block=16, e4m3=e4m3), [16 * 9], hkv=1, d=64)
        x = torch.randn((9, 16, 64), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
        x[0] = 0.0
        x[1] *= 2.0 ** -100
        x[2, 3, 5], x[2, 3, 6] = math.inf, -math.inf
        x[3, 7] = math.nan
        x[4] = 127.0
        x[5, 2, 2] = -127.5
        x[6] = 3.3e38
        x[7] = 2.0 ** -133
        x[8] = -2.0 ** -80 * 127
        for r in range(16 * 9):
            page, hh, i = pool.place(0, 0, [r])
            at = (int(page), hh, int(i))
            if e4m3:
                (pool.k[at],), (pool.k_scale[at],) = (y.cuda() for y in ref.e4m3_rows(x.view(-1, 64)[r][None]))
            else:
                pool.k[at] = x.view(-1, 64)[r].to(BF16).cuda()
        _summarize(pool, blocks, None, 16 * 9, [2])


def test_summarize_leaves_blocks_without_a_page_out():
    pool, blocks = _pool(dict(page_rows=32, block=16), [200, 200])
    pool.table[0, 1], pool.table[1, 0], pool.table[1, 4] = -1, pool.n_pages, -2 ** 31
    _summarize(pool, blocks, None, 200, [2, 2])


# ---- choice ----------------------------------------------------------------------------------------
def _random_bounds(pool, blocks, seed=3):
    g = torch.Generator().manual_seed(seed)
    a = torch.randint(-127, 128, blocks.bounds.shape, generator=g).to(torch.int8)
    hi, lo = a.amax(3), a.amin(3)
    blocks.bounds.copy_(torch.stack([hi, lo], 3))
    blocks.scale.copy_(torch.randint(118, 126, blocks.scale.shape, generator=g))


def _choose(pool, blocks, new, n_chosen, first, recent, *, hq, policy=None, max_rows=None, cu=True, q=None, total=None, seed=2):
    policy = policy or [2] * pool.H
    sums = _sums(new)
    total = total or max(1, sums[-1])
    if q is None:
        q = torch.randn((total, hq, pool.D), generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()
    cfg, most = _cfg(pool, hq, policy), max_rows or pool.max_pages * pool.R
    n_past = sum(p >> 1 for p in policy)
    out = torch.full((total, n_past, n_chosen), -7, dtype=I32, device="cuda")
    need = sa.seg_kv_paged_choose_workspace_bytes(cfg, pool.pages(), blocks.c, total, most, n_chosen)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_choose(cfg, pool.pages(), blocks.c, q, torch.tensor(sums, dtype=I32, device="cuda") if cu else None, total, max(1, max(new)),
                           pool.rows, most, n_chosen, first, recent, out, ws, need, stream=_stream())
    want = sref.chosen(pool, blocks, q, sums, _list(pool), policy, n_chosen, first, recent, max_rows)
    assert torch.equal(out.cpu(), want)
    return out


@pytest.mark.parametrize("kind", BLOCKS[:4], ids=_name)
@pytest.mark.parametrize("d,g", [(128, 4), (64, 1)])
def test_choose_for_one_token_each(kind, d, g):
    pool, blocks = _pool(kind, [0, 1, 64, 65, [500, 130], 900], d=d)
    _random_bounds(pool, blocks)
    for n_chosen, first, recent in ((1, 0, 1), (5, 1, 2), (6, 0, 6), (9, 4, 1)):
        _choose(pool, blocks, [1] * 6, n_chosen, first, recent, hq=2 * g, cu=None)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 8, 13, 16, 17, 40, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_choose_for_any_group_and_ragged_tokens(g, d):
    pool, blocks = _pool(dict(page_rows=32, block=16), [300, 40, 0, [410, 205]], d=d)
    _random_bounds(pool, blocks)
    _choose(pool, blocks, [19, 3, 0, 6], 7, 1, 2, hq=2 * g, policy=[2, 3], total=35)


def test_choose_between_equal_scores_takes_the_lower_block():
    pool, blocks = _pool(dict(page_rows=64, block=16), [4000], hkv=1)
    _random_bounds(pool, blocks)
    blocks.bounds[:] = blocks.bounds[0, 0, 0]
    blocks.scale[:] = 120
    _choose(pool, blocks, [1], 50, 2, 3, hq=4)
    blocks.scale[::2] = 121
    _choose(pool, blocks, [1], 50, 2, 3, hq=4)
    _choose(pool, blocks, [1], 200, 2, 3, hq=4)
    _choose(pool, blocks, [1], 9, 0, 1, hq=4, q=torch.zeros((1, 4, 128), dtype=BF16, device="cuda"))


def test_choose_with_extreme_scales_and_queries():
    pool, blocks = _pool(dict(page_rows=64, block=16), [3000], hkv=2)
    _random_bounds(pool, blocks)
    blocks.scale.copy_(torch.randint(47, 250, blocks.scale.shape, generator=torch.Generator().manual_seed(1)))
    blocks.bounds[3], blocks.bounds[5] = 127, -127
    q = torch.randn((5, 8, 128), generator=torch.Generator().manual_seed(2))
    q[0] *= 1e-38
    q[1] *= 1e37
    q[2, 3, 7], q[2, 5, 8], q[2, 1] = math.inf, math.nan, -math.inf
    q[3] = 127.0
    q[4] = 255.0 / 2 ** 130
    _choose(pool, blocks, [5], 20, 1, 1, hq=8, q=q.to(BF16).cuda())


def test_choose_takes_blocks_without_a_page_last():
    pool, blocks = _pool(dict(page_rows=32, block=16), [600, 600])
    _random_bounds(pool, blocks)
    pool.table[0, 1:9], pool.table[1, 0], pool.table[1, 18] = -1, pool.n_pages, -1
    _choose(pool, blocks, [1, 3], 12, 1, 2, hq=4)
    _choose(pool, blocks, [1, 3], 30, 1, 2, hq=4)


def test_choose_among_many_blocks_and_up_to_max_rows():
    pool, blocks = _pool(dict(page_rows=256, block=16), [60000], hkv=1, d=64)
    _random_bounds(pool, blocks)
    for n_chosen in (1, 64, 3000):
        _choose(pool, blocks, [2], n_chosen, 0, 1, hq=2)
    _choose(pool, blocks, [2], 40, 3, 4, hq=2, max_rows=33333)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_choose_for_chunks_behind_many_blocks(d, g):
    """Tokens that share the bounds they are scored with, in tiles that end amid sequences and hold several."""
    new = [70, 3, 0, 130, 5, 1]
    pool, blocks = _pool(dict(page_rows=64, block=16), [5000, 5200, 4000, 900, 4777, 4200], d=d, hkv=2)
    _random_bounds(pool, blocks)
    _choose(pool, blocks, new, 24, 1, 2, hq=2 * g, policy=[2, 3], total=sum(new) + 3)


def test_choose_in_parts_of_the_tokens():
    """More keys than the workspace holds at a time: the tokens go in parts."""
    pool, blocks = _pool(dict(page_rows=16, block=16), [3000], hkv=1, d=64)
    _random_bounds(pool, blocks)
    cfg = _cfg(pool, 1)
    n, most = 2500, pool.max_pages * pool.R
    # a table with room for far more rows than are held makes every token's keys long
    wide = torch.full((1, 4_000_000 // 16), -1, dtype=I32, device="cuda")
    wide[:, :pool.max_pages] = pool.table
    pages = sa.make_pages(k=pool.k, v=pool.v, table=wide, max_pages=wide.shape[1], page_rows=16, n_pages=pool.n_pages)
    q = torch.randn((n, 1, 64), generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    cu = torch.tensor([0, n], dtype=I32, device="cuda")
    got = []
    for p, rows in ((pool.pages(), most), (pages, 4_000_000)):
        need = sa.seg_kv_paged_choose_workspace_bytes(cfg, p, blocks.c, n, rows, 9)
        assert need <= 300 << 20
        assert (need < n * 4 * -(-rows // 16)) == (rows == 4_000_000)
        out = torch.full((n, 1, 9), -7, dtype=I32, device="cuda")
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        sa.seg_kv_paged_choose(cfg, p, blocks.c, q, cu, n, n, pool.rows, rows, 9, 1, 1, out, ws, need, stream=_stream())
        got.append(out)
    assert torch.equal(*got) and (got[0] != -7).all()


# ---- attention -------------------------------------------------------------------------------------
def _lists(pool, new, n_chosen, block, policy, seed=4, total=None):
    """Lists of the caller's own: any order, entries that are none, one behind the token's block."""
    g = torch.Generator().manual_seed(seed)
    sums = _sums(new)
    n_past = sum(p >> 1 for p in policy)
    out = torch.full((total or max(1, sums[-1]), n_past, n_chosen), -1, dtype=I32)
    past = [h for h in range(pool.H) if policy[h] & 2]
    for b, m in enumerate(new):
        for i in range(m):
            for x, h in enumerate(past):
                own = max(0, int(pool.rows[b, h]) - m + i) // block
                row = torch.randperm(own + 2, generator=g)[:n_chosen].to(I32)
                out[sums[b] + i, x, :len(row)] = row
                if n_chosen > 2:
                    out[sums[b] + i, x, 1] = -5
    return out


def _attend(pool, block, new, n_chosen, *, hq, policy=None, seg=64, tail=16, out_fp32=True, max_rows=None, cu=True, q=None, total=None, scale=0.0, lists=None):
    policy = policy or [2] * pool.H
    sums = _sums(new)
    total = total or max(1, sums[-1])
    if q is None:
        q = torch.randn((total, hq, pool.D), generator=torch.Generator().manual_seed(8)).to(BF16).cuda()
    lists = _lists(pool, new, n_chosen, block, policy, total=total) if lists is None else lists
    cfg, most = _cfg(pool, hq, policy, seg, tail, out_fp32=out_fp32, scale=scale), max_rows or pool.max_pages * pool.R
    out = torch.full((total, hq, pool.D), 77.0, dtype=torch.float32 if out_fp32 else BF16, device="cuda")
    lse = torch.full((total, hq), 77.0, device="cuda")
    blocks = sa.make_blocks(block_rows=block)
    need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, total, max(1, max(new)), most, n_chosen)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_attn_paged_chosen(cfg, pool.pages(), blocks, q, torch.tensor(sums, dtype=I32, device="cuda") if cu else None, total, max(1, max(new)), pool.rows,
                             most, lists.cuda() if lists.numel() else None, n_chosen, out, lse, ws, need, stream=_stream())
    torch.cuda.synchronize()
    want, want_lse, odd, most_s, most_v = sref.attention(pool, q, sums, _list(pool), policy, seg, tail, lists, block, scale, max_rows)
    assert (out[sums[-1]:] == 77.0).all() and (lse[sums[-1]:] == 77.0).all()
    out, lse, want, want_lse, odd = out[:sums[-1]].double().cpu(), lse[:sums[-1]].double().cpu(), want[:sums[-1]], want_lse[:sums[-1]], odd[:sums[-1]]
    # A score is a sum of D exact products in fp32: off by D 2^-24 of the sum of their magnitudes at most.  A weight adds the
    # rounding of its argument, of exp2 and of the sums: 2^-20.  What the split weights lose: 2^-16 of a weight.
    delta = pool.D * 2.0 ** -24 * most_s + 2.0 ** -20
    half = 0.0 if out_fp32 else 2.0 ** -8 * (1 + 2.0 ** -7)
    err, bound = (out - want).abs(), want.abs() * half + (2 * delta + 2.0 ** -16) * most_v
    assert ((err <= bound) | odd[..., None]).all(), f"out: {float((err - bound)[~odd].max()):.3e} above the bound"
    empty = want_lse == -math.inf
    assert torch.equal((lse == -math.inf)[~odd], empty[~odd])
    err = (lse - want_lse)[~empty & ~odd].abs()
    assert (err <= delta + 2.0 ** -22 * (1 + want_lse[~empty & ~odd].abs())).all(), f"lse: {float(err.max()):.3e}"
    return out, lse, odd


KINDS = BLOCKS + [dict(page_rows=256, block=128)]


@pytest.mark.parametrize("kind", KINDS, ids=_name)
@pytest.mark.parametrize("d,g", [(128, 4), (64, 1)])
def test_attention_of_one_token_each(kind, d, g):
    pool, blocks = _pool(kind, [0, 1, 31, 33, [129, 64], 517], d=d)
    _attend(pool, blocks.rows, [1] * 6, 6, hq=2 * g, policy=[2, 1], cu=None)
    _attend(pool, blocks.rows, [1] * 6, 3, hq=2 * g, policy=[0, 3])


@pytest.mark.parametrize("kind", KINDS, ids=_name)
@pytest.mark.parametrize("d,g", [(128, 4), (64, 3)])
def test_attention_of_ragged_tokens(kind, d, g):
    pool, blocks = _pool(kind, [40, 0, [200, 150, 200], 3, 7], d=d, hkv=3)
    _attend(pool, blocks.rows, [40, 0, 77, 3, 1], 5, hq=3 * g, policy=[2, 1, 0], total=130)


@pytest.mark.parametrize("g", [1, 2, 5, 8, 16, 17, 40, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_any_group(g, d):
    pool, blocks = _pool(dict(page_rows=32, block=16), [100, 37], d=d)
    _attend(pool, 16, [9, 2], 4, hq=2 * g, policy=[2, 1], seg=32, tail=8)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("out_fp32", [False, True])
def test_attention_of_long_histories_in_parts(e4m3, out_fp32):
    """One sequence: windows are shared out among workgroups and joined."""
    pool, _ = _pool(dict(page_rows=128, block=64, e4m3=e4m3), [9001], hkv=2)
    _attend(pool, 64, [1], 70, hq=8, policy=[2, 1], seg=4096, tail=1024, out_fp32=out_fp32, cu=None)
    _attend(pool, 64, [3], 70, hq=8, policy=[2, 1], seg=4096, tail=1024, out_fp32=out_fp32, max_rows=8999, scale=0.21)


def test_attention_of_windows_only():
    pool, _ = _pool(dict(page_rows=16, block=16), [300, 90, 0])
    _attend(pool, 16, [200, 90, 0], 1, hq=4, policy=[1, 0], lists=torch.empty(0), total=300)


def test_attention_without_a_row():
    pool, _ = _pool(dict(page_rows=16, block=16), [70, 70])
    lists = torch.full((4, 1, 3), -1, dtype=I32)
    lists[1, 0] = torch.tensor([5, 2 ** 31 - 1, -2 ** 31])
    pool.table[1, 4] = -1
    _attend(pool, 16, [2, 2], 3, hq=4, policy=[2, 0], lists=lists)


def test_attention_counts_a_block_that_is_listed_twice_twice():
    pool, _ = _pool(dict(page_rows=48, block=48), [400], hkv=1)
    _attend(pool, 48, [1], 5, hq=4, lists=torch.tensor([[[7, 7, 3, 7, 3]]], dtype=I32))


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_is_not_touched_by_rows_that_are_not_seen(e4m3):
    """Rows of NaN: in blocks that are not listed, behind the token's own, before a window, and in a chunk between its tokens."""
    pool, _ = _pool(dict(page_rows=32, block=32, e4m3=e4m3), [260], hkv=2)
    for r in (33, 40, 200, 230, 233, 239):
        for h in range(2):
            page, hh, i = pool.place(0, h, [r])
            for x in (pool.k, pool.v):
                x[page.cuda(), hh, i.cuda()] = 0x7F if e4m3 else math.nan
    lists = torch.tensor([0, 2, 4, 6, 7, 8], dtype=I32).repeat(61, 1, 1)
    out, lse, odd = _attend(pool, 32, [61], 6, hq=8, policy=[2, 1], lists=lists)
    assert not odd.all() and odd.any() and out[~odd].isfinite().all()
    for inf in (math.inf, -math.inf) if not e4m3 else ():
        pool, _ = _pool(dict(page_rows=32, block=32), [260], hkv=2)
        page, hh, i = pool.place(0, 1, [231])
        pool.v[page.cuda(), hh, i.cuda(), 5] = inf
        out, lse, odd = _attend(pool, 32, [61], 6, hq=8, policy=[2, 1], lists=lists)
        assert odd.any() and out[~odd].isfinite().all()


@pytest.mark.parametrize("kind", KINDS, ids=_name)
def test_attention_of_ragged_tokens_in_bf16(kind):
    pool, blocks = _pool(kind, [150, 33, [90, 300, 200]], hkv=3)
    _attend(pool, blocks.rows, [150, 2, 64], 4, hq=12, policy=[1, 2, 3], seg=100, tail=7, out_fp32=False)


# Tokens so many that their windows share tiles, in windows long enough to be cut into many pieces: the start of a segment amid the tokens of a piece,
# sequences without tokens, with one and without a row before.
SHARED = [(dict(page_rows=64, block=64), 128, 4, True), (dict(page_rows=128, block=64, per_head=True, e4m3=True), 128, 4, False),
          (dict(page_rows=48, block=48, token_major=True), 64, 4, True), (dict(page_rows=80, block=80, e4m3=True), 64, 1, True),
          (dict(page_rows=64, block=64), 128, 16, False), (dict(page_rows=32, block=16, per_head=True), 128, 3, True)]


@pytest.mark.parametrize("kind,d,g,out_fp32", SHARED, ids=range(len(SHARED)))
def test_attention_of_windows_that_share_tiles(kind, d, g, out_fp32):
    new, held = [900, 1100, 0, 1], [1990, 3500, 100, 0]
    pool, blocks = _pool(kind, [h + n for h, n in zip(held, new)], d=d, hkv=3)
    _attend(pool, blocks.rows, new, 4, hq=3 * g, policy=[1, 2, 0], seg=1000, tail=300, total=sum(new) + 2, out_fp32=out_fp32)


@pytest.mark.parametrize("e4m3", [False, True])
def test_windows_that_share_tiles_are_not_touched_by_rows_that_are_not_seen(e4m3):
    """NaN before every window and before some, behind tokens' own rows, at a segment's start, in a row without a page; infinities in one channel."""
    for odd_row in ((100, 690, 1000, 2100, 2800, 3499), (1990, 2999)):
        pool, _ = _pool(dict(page_rows=32, block=32, e4m3=e4m3), [3500], hkv=3)
        for r in odd_row:
            for h in range(3):
                page, hh, i = pool.place(0, h, [r])
                for x in (pool.k, pool.v) if len(odd_row) > 2 else (pool.v,):
                    if e4m3 or len(odd_row) > 2:
                        x[page.cuda(), hh, i.cuda()] = 0x7F if e4m3 else math.nan
                    else:
                        x[page.cuda(), hh, i.cuda(), 7] = math.inf if r == 2999 else -math.inf
        pool.table[0, 1600 // 32] = -1
        out, lse, odd = _attend(pool, 32, [2000], 3, hq=12, policy=[1, 2, 0], seg=1000, tail=300)
        assert not odd.all() and odd.any() and out[~odd].isfinite().all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_of_windows_with_a_workgroup_each(e4m3):
    """So many tokens and heads that windows are not cut: 2064 times eight tokens in one head's window."""
    new, held = [2044, 6], [130, 0]
    pool, blocks = _pool(dict(page_rows=64, block=64, e4m3=e4m3), [h + n for h, n in zip(held, new)], hkv=8)
    _attend(pool, blocks.rows, new, 1, hq=128, policy=[1, 0, 1, 1, 0, 0, 1, 1], seg=200, tail=56, out_fp32=not e4m3)


def test_attention_of_lists_in_parts_of_the_tokens():
    """More partials than the workspace holds at a time: the tokens go in parts, to the same results as in calls of their own."""
    pool, _ = _pool(dict(page_rows=256, block=64), [9000], hkv=1)
    n, chosen, most, hq = 8400, 72, pool.max_pages * pool.R, 4
    g = torch.Generator().manual_seed(8)
    q = torch.randn((n, hq, 128), generator=g).to(BF16).cuda()
    lists = torch.randint(0, 9000 // 64 + 2, (n, 1, chosen), generator=g).to(I32)
    cfg, blocks = _cfg(pool, hq), sa.make_blocks(block_rows=64)
    entry = hq * (128 + 2) * 4  # bytes of an entry's partials
    assert n * chosen * entry > sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, n, n, most, chosen) > 5000 * chosen * entry

    def call(first, count):
        out, lse = torch.empty((count, hq, 128), dtype=BF16, device="cuda"), torch.empty((count, hq), device="cuda")
        rows = torch.tensor([[9000 - (n - first - count)]], dtype=I32, device="cuda")
        need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, count, count, most, chosen)
        assert need > count * chosen * entry or count == n
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        sa.seg_attn_paged_chosen(cfg, pool.pages(), blocks, q[first:first + count].contiguous(), torch.tensor([0, count], dtype=I32, device="cuda"), count, count,
                                 rows, most, lists[first:first + count].cuda(), chosen, out, lse, ws, need, stream=_stream())
        return out, lse

    out, lse = call(0, n)
    parts = [call(0, 3000), call(3000, 3000), call(6000, 2400)]
    assert torch.equal(out, torch.cat([p[0] for p in parts])) and torch.equal(lse, torch.cat([p[1] for p in parts]))
    # and the last tokens against the definition
    last = 5
    want, want_lse, _, most_s, most_v = sref.attention(pool, q[-last:], [0, last], [[9000]], [2], 64, 16, lists[-last:], 64)
    delta = 128 * 2.0 ** -24 * most_s + 2.0 ** -20
    assert ((out[-last:].double().cpu() - want).abs() <= want.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + (2 * delta + 2.0 ** -16) * most_v).all()
    assert ((lse[-last:].double().cpu() - want_lse).abs() <= delta + 2.0 ** -22 * (1 + want_lse.abs())).all()


# Chunks so long that a listed block is taken once for all tokens that list it.
def _long_chunk(kind, *, d=128, g=4, policy=(2, 3), chosen=8, new=(1290, 0, 17), held=(700, 30, 2000), seed=0):
    lengths = [h + n for h, n in zip(held, new)]
    pool, blocks = _pool(kind, lengths, d=d, hkv=len(policy), seed=seed)
    total = sum(new) + 3
    cfg, most = _cfg(pool, len(policy) * g, list(policy)), pool.max_pages * pool.R
    need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), sa.make_blocks(block_rows=blocks.rows), total, max(new), most, chosen)
    assert need > sum(new) * 2 * chosen * g * d * 4  # the partials of every entry
    return pool, blocks.rows, list(new), total


LONG = [dict(page_rows=64, block=64), dict(page_rows=128, block=128, per_head=True), dict(page_rows=96, block=48), dict(page_rows=80, block=80, token_major=True),
        dict(page_rows=64, block=64, e4m3=True), dict(page_rows=128, block=64, e4m3=True, per_head=True)]


@pytest.mark.parametrize("kind", LONG, ids=_name)
@pytest.mark.parametrize("out_fp32", [False, True])
def test_attention_of_long_chunks(kind, out_fp32):
    chosen, g = (16, 2) if kind.get("e4m3") else (8, 4)
    pool, block, new, total = _long_chunk(kind, chosen=chosen, g=g, **(dict(new=(2600, 0, 17)) if kind.get("e4m3") else {}))
    _attend(pool, block, new, chosen, hq=2 * g, policy=[2, 3], out_fp32=out_fp32, total=total)


@pytest.mark.parametrize("d,g", [(64, 1), (64, 8), (128, 3), (128, 1)])
def test_attention_of_long_chunks_of_any_group(d, g):
    chosen = 16 if g == 8 else 8
    pool, block, new, total = _long_chunk(dict(page_rows=64, block=64), d=d, g=g, chosen=chosen, new=(2600, 0, 17) if g == 8 else (1290, 0, 17))
    _attend(pool, block, new, chosen, hq=2 * g, policy=[2, 3], total=total)


def test_long_chunks_repeat_bit_for_bit_and_replay():
    """The order in which listed blocks' entries are gathered is not that of the results; two graphs with a workspace each, lists that change."""
    chosen, g = 8, 4
    pool, block, new, total = _long_chunk(dict(page_rows=64, block=64), chosen=chosen, g=g)
    cfg, blocks, most = _cfg(pool, 2 * g, [2, 3]), sa.make_blocks(block_rows=block), pool.max_pages * pool.R
    q = torch.randn((total, 2 * g, 128), generator=torch.Generator().manual_seed(8)).to(BF16).cuda()
    cu = torch.tensor(_sums(new), dtype=I32, device="cuda")
    need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, total, max(new), most, chosen)
    lists = _lists(pool, new, chosen, block, [2, 3], total=total).cuda()
    sides = [(torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), torch.zeros((total, 2 * g, 128), device="cuda").to(BF16),
              torch.zeros((total, 2 * g), device="cuda")) for _ in range(3)]

    def call(ws, out, lse):
        sa.seg_attn_paged_chosen(cfg, pool.pages(), blocks, q, cu, total, max(new), pool.rows, most, lists, chosen, out, lse, ws, need, stream=_stream())

    call(*sides[0])
    torch.cuda.synchronize()
    graphs = []
    for side in sides[1:]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(*side)
    for i in range(4):
        lists.copy_(_lists(pool, new, chosen, block, [2, 3], seed=20 + i, total=total))
        call(*sides[0])
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for graph, s in zip(graphs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for side in sides[1:]:
            assert torch.equal(side[1], sides[0][1]) and torch.equal(side[2], sides[0][2])
        before = [x.clone() for x in sides[0][1:]]
        call(*sides[0])
        assert all(torch.equal(x, y) for x, y in zip(before, sides[0][1:]))


@pytest.mark.parametrize("e4m3", [False, True])
def test_long_chunks_are_not_touched_by_rows_that_are_not_seen(e4m3):
    """NaN in blocks that some tokens do not list, behind tokens' own rows in blocks that they do, in rows without a page."""
    n, chosen, g = (2600, 16, 2) if e4m3 else (1400, 8, 4)
    pool, block, new, total = _long_chunk(dict(page_rows=64, block=64, e4m3=e4m3), new=(n, 0, 0), held=(600, 0, 0), chosen=chosen, g=g)
    for r in (70, 71, 900, 1203, 1255, 1999):
        for h in range(2):
            page, hh, i = pool.place(0, h, [r])
            for x in (pool.k, pool.v):
                x[page.cuda(), hh, i.cuda()] = 0x7F if e4m3 else math.nan
    pool.table[0, 5] = -1
    lists = _lists(pool, new, chosen, block, [2, 3], total=total)
    own = (600 + torch.arange(n)) // 64
    lists[:n, :, 0] = own[:, None].to(I32)
    out, lse, odd = _attend(pool, block, new, chosen, hq=2 * g, policy=[2, 3], lists=lists, total=total)
    assert not odd.all() and odd.any() and out[~odd].isfinite().all()
