"""Forms of the sparse attention's operators that only calls of certain sizes take (test_chosen_forms.py: that these do): the selections of blocks
for hundreds and thousands of lists, reservations by several launches, windows of many short sequences and of segments shorter than a workgroup's tokens."""
import pytest
import torch

import paper_2605_11744_amd as sa
import sparse_ref as sref
from paged_ref import Pool
from test_gpu_sparse import BF16, I32, P3, Tables, _attend, _cfg, _list, _lists, _random_bounds, _stream, _sums

pytestmark = pytest.mark.gpu
F64 = torch.float64


# ---- choice ----------------------------------------------------------------------------------------
def _chosen_at_once(pool, blocks, q, cu, n_chosen, first, recent):
    """sref.chosen for all tokens of a sequence together: whole numbers below 2^53 in 64-bit floats, times powers of two."""
    bounds, scale = blocks.bounds.cpu().to(F64), blocks.scale.cpu().to(F64)
    out = torch.full((q.shape[0], pool.H, n_chosen), -7, dtype=I32)
    g = q.shape[1] // pool.H
    for b in range(pool.B):
        m = cu[b + 1] - cu[b]
        for h in range(pool.H if m else 0):
            rows = int(pool.rows[b, h])
            n = max(0, rows - 1) // blocks.rows + 1
            page, hh, r = pool.place(b, h, torch.arange(n) * blocks.rows)
            at = page.clamp(min=0), hh, r // blocks.rows
            group = q[cu[b]:cu[b + 1], h * g:(h + 1) * g].to(F64).cpu()
            most = group.abs().amax((1, 2))
            e = torch.tensor([sref.least_exponent(float(x)) or 0 for x in most], dtype=F64)
            q8 = (group * torch.exp2(-e)[:, None, None]).round()
            dot = torch.einsum("tgd,jd->tgj", q8.clamp(min=0), bounds[at][:, 0]) + torch.einsum("tgd,jd->tgj", q8.clamp(max=0), bounds[at][:, 1])
            score = dot.amax(1) * torch.exp2(scale[at] - 127)
            score[:, page < 0] = -torch.inf
            for i in range(m):
                own = max(0, rows - m + i) // blocks.rows if rows - m + i >= 0 else -1
                if own + 1 <= n_chosen:
                    got = list(range(own + 1))
                else:
                    # (a stable sort: among equals the lower block)
                    picks = score[i, first:own - recent + 1].sort(descending=True, stable=True)[1][:n_chosen - first - recent] + first
                    got = sorted([*range(first), *picks.tolist(), *range(own - recent + 1, own + 1)])
                out[cu[b] + i, h] = torch.tensor(got + [-1] * (n_chosen - len(got)), dtype=I32)
    return out


# New tokens, rows before them, blocks of 16 rows in all; two heads' lists: 512 to 4095 of them have a workgroup each, from 4096 on a wave each, with
# more keys than its registers hold
SELECTIONS = [([290, 0, 13], [4400, 300, 8200]), ([300], [33000]), ([2000, 60, 0, 5], [4500, 5000, 70, 4200]), ([2050], [17000])]


@pytest.mark.parametrize("ties", [False, True], ids=["distinct", "ties"])
@pytest.mark.parametrize("new,held", SELECTIONS)
def test_selections_of_many_lists(new, held, ties):
    pool = Pool(batch=len(new), hkv=2, d=64, page_rows=64, max_pages=-(-max(h + n for h, n in zip(held, new)) // 64)).fill([0] * len(new))
    pool.rows.copy_(torch.tensor([[h + n] * 2 for h, n in zip(held, new)], dtype=I32))  # (no call here reads keys)
    blocks = sref.Blocks(pool, 16)
    _random_bounds(pool, blocks)
    if ties:  # few scores: a block's bounds are one of four kinds
        kinds = torch.randint(0, 4, blocks.scale.shape, generator=torch.Generator().manual_seed(4))
        blocks.bounds.copy_(blocks.bounds[0, 0, 0].cpu() * (kinds[..., None, None] // 2) // 2)
        blocks.scale.copy_(118 + kinds % 2)
    pool.table[0, 3] = -1
    sums, total = _sums(new), sum(new) + (2 if len(new) > 1 else 0)
    assert (total * 2 >= 512) and (total * 2 >= 4096) == (max(new) >= 2000)
    q = torch.randn((total, 4, 64), generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    cfg, most = _cfg(pool, 4), pool.max_pages * 64
    for n_chosen, first, recent in ((24, 1, 2), (100, 0, 1)):
        out = torch.full((total, 2, n_chosen), -7, dtype=I32, device="cuda")
        need = sa.seg_kv_paged_choose_workspace_bytes(cfg, pool.pages(), blocks.c, total, most, n_chosen)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        sa.seg_kv_paged_choose(cfg, pool.pages(), blocks.c, q, torch.tensor(sums, dtype=I32, device="cuda"), total, max(new), pool.rows, most, n_chosen, first,
                               recent, out, ws, need, stream=_stream())
        want = _chosen_at_once(pool, blocks, q, sums, n_chosen, first, recent)
        assert torch.equal(out.cpu(), want)
        # the plain form agrees, where it is quick enough to be asked: the last token of the first sequence
        t = new[0] - 1
        one = sref.chosen(pool, blocks, q[t:t + 1], [0] + [1] * len(new), _list(pool), [2, 2], n_chosen, first, recent)
        assert torch.equal(one[0], want[t])


# ---- tables ----------------------------------------------------------------------------------------
def _many(per_head, n, most, seed, page_rows=16):
    g = torch.Generator().manual_seed(seed)
    rows = torch.randint(0, 200, (n, 3), generator=g).tolist()
    new = torch.randint(0, most + 1, (n,), generator=g).tolist()
    need = sum(-(-(200 + m) // page_rows) for m in new) * (3 if per_head else 1)
    t = Tables(rows=rows, page_rows=page_rows, max_pages=(200 + most) // page_rows + 1, per_head=per_head, policy=P3, n_pages=need + 2 * n, seed=seed)
    return t, new


# (sequences, most new tokens of one): one workgroup, several launches, and more sequences than the threads of one of theirs
RESERVATIONS = [(200, 2), (60, 300), (700, 3), (1100, 40)]


@pytest.mark.parametrize("newest", [False, True], ids=["all", "newest"])
@pytest.mark.parametrize("per_head", [False, True], ids=["shared", "per_head"])
@pytest.mark.parametrize("n,most", RESERVATIONS)
def test_reserve_for_many_sequences(n, most, per_head, newest):
    """With pages for all, and with so few that a sequence in the middle is the first that gets none, and some behind it that need none still do."""
    t, new = _many(per_head, n, most, n)
    free = int((t.users <= 0).sum())
    table, users, granted, _ = t.reserve(new, newest)
    assert granted == [1] * n
    taken = int((users > 0).sum() - (t.users > 0).sum())
    assert 10 < taken < free
    t.take_away(taken // 2)
    granted = t.reserve(new, newest)[2]
    assert 0 < sum(granted) < n


def test_both_ways_of_reserving_give_the_same():
    """A pool of 2^18 pages and one of a page more."""
    got = []
    for n_pages in (1 << 18, (1 << 18) + 1):
        rows = [[i * 7, 300 - i, 64] for i in range(40)]
        t = Tables(rows=rows, page_rows=16, max_pages=30, policy=P3, n_pages=9000, seed=3)
        taken = torch.ones(n_pages, dtype=I32)
        taken[-600:-6] = 0
        t.table[t.table >= 0] += n_pages - 9000 - 700  # (anywhere but among the free ones)
        t.n_pages, t.users = n_pages, taken
        got.append(t.reserve([1 + i % 3 for i in range(40)])[:3])
    a, b = got
    shift = 1
    moved = torch.where(a[0] >= 0, a[0] + shift, a[0])
    assert torch.equal(moved, b[0]) and a[2] == b[2]


# ---- attention -------------------------------------------------------------------------------------
def _short_sequences(n, most, seed):
    g = torch.Generator().manual_seed(seed)
    new = torch.randint(0, most + 1, (n,), generator=g)
    new[::5] = 0
    return new.tolist(), torch.randint(0, 60, (n,), generator=g).tolist()


# d, g, policy, segment, tail, (new tokens, rows before them), how the windows are taken.  A unit is 128 / g neighbouring tokens of a sequence.
SHORT = [(64, 1, [1, 0], 32, 8, ([6000], [10]), "shares"),                              # five segments' starts amid a unit
         (128, 2, [1, 2, 0], 20, 20, ([4000, 0, 1500], [0, 5, 33]), "shares"),         # a window is shorter than a unit
         (64, 1, [1, 0, 1, 0], 16, 8, _short_sequences(300, 40, 1), "shares"),          # hundreds of sequences, many of them without tokens
         (128, 1, [1, 0, 1, 1, 0, 0, 1, 0], 16, 8, _short_sequences(300, 32, 2), "units"),
         (64, 1, [0] * 8, 1, 0, ([9000], [0]), "shares")]                               # a token sees itself


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("d,g,policy,seg,tail,batch,_", SHORT, ids=range(len(SHORT)))
def test_windows_of_short_segments_and_sequences(d, g, policy, seg, tail, batch, _, e4m3):
    new, held = batch
    pool = Pool(batch=len(new), hkv=len(policy), d=d, page_rows=16, max_pages=-(-max(h + n for h, n in zip(held, new)) // 16), e4m3=e4m3)
    pool.fill([h + n for h, n in zip(held, new)])
    lists = None if 2 in policy else torch.empty(0)
    _attend(pool, 16, new, 4, hq=g * len(policy), policy=policy, seg=seg, tail=tail, out_fp32=not e4m3, total=sum(new) + (len(new) > 1), lists=lists)


def test_one_workspace_for_all_calls_of_a_program():
    """Asked for the largest chunk; smaller ones and steps, which take other forms, give in it what they give in one of their own."""
    pool = Pool(batch=2, hkv=2, d=128, page_rows=64, max_pages=60).fill([3000, 3600])
    policy, hq, block, chosen = [2, 1], 8, 64, 16
    cfg, blocks, most = _cfg(pool, hq, policy, 1000, 300), sa.make_blocks(block_rows=block), pool.max_pages * pool.R
    bytes_of = lambda total, longest: sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, total, longest, most, chosen)
    shared = torch.full((bytes_of(2800, 1600),), 0xFF, dtype=torch.uint8, device="cuda")
    for new in ([1200, 1600], [1, 1], [400, 3], [2, 5], [0, 1], [64, 64]):
        total, longest = sum(new), max(new)
        q = torch.randn((total, hq, 128), generator=torch.Generator().manual_seed(total)).to(BF16).cuda()
        lists, cu = _lists(pool, new, chosen, block, policy).cuda(), torch.tensor(_sums(new), dtype=I32, device="cuda")
        need = bytes_of(total, longest)
        assert need <= shared.numel()
        got = []
        for ws in (shared, torch.full((need,), 0x11, dtype=torch.uint8, device="cuda"), shared):
            out, lse = torch.empty((total, hq, 128), dtype=BF16, device="cuda"), torch.empty((total, hq), device="cuda")
            sa.seg_attn_paged_chosen(cfg, pool.pages(), blocks, q, cu, total, longest, pool.rows, most, lists, chosen, out, lse, ws, ws.numel(), stream=_stream())
            got.append((out, lse))
        assert all(torch.equal(got[0][i], x[i]) for x in got[1:] for i in (0, 1)), new


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_step_of_one_sequence_repeats_bit_for_bit(e4m3):
    """Lists and windows shared out among workgroups and joined."""
    pool = Pool(batch=1, hkv=4, d=128, page_rows=64, max_pages=330, e4m3=e4m3).fill([21000])
    policy, hq, chosen = [2, 1, 3, 0], 16, 64
    cfg, blocks, most = _cfg(pool, hq, policy, 4096, 1024, out_fp32=True), sa.make_blocks(block_rows=64), pool.max_pages * pool.R
    q, lists = torch.randn((1, hq, 128), generator=torch.Generator().manual_seed(1)).to(BF16).cuda(), _lists(pool, [1], chosen, 64, policy).cuda()
    need = sa.seg_attn_paged_chosen_workspace_bytes(cfg, pool.pages(), blocks, 1, 1, most, chosen)
    got = []
    for fill in (0x00, 0xFF, 0x11):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        out, lse = torch.empty((1, hq, 128), device="cuda"), torch.empty((1, hq), device="cuda")
        sa.seg_attn_paged_chosen(cfg, pool.pages(), blocks, q, None, 1, 1, pool.rows, most, lists, chosen, out, lse, ws, need, stream=_stream())
        got.append((out, lse))
    assert all(torch.equal(got[0][i], x[i]) for x in got[1:] for i in (0, 1))
