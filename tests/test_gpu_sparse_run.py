"""Sparse attention over a paged cache as a program runs it: pages reserved, tokens appended, bounds formed, blocks chosen, attended to, rows
evicted, pages released -- call after call, captured and replayed, on streams of their own."""
import math

import pytest
import torch

import paper_2605_11744_amd as sa
import sparse_ref as sref
from paged_ref import Pool, bits

pytestmark = pytest.mark.gpu
BF16, I32, I64 = torch.bfloat16, torch.int32, torch.int64
SEG, TAIL, POLICY, HQ, D = 64, 16, [2, 1, 3], 6, 64


class Program:
    """A pool whose tables are kept on the GPU, and the buffers of its steps."""

    def __init__(self, batch, *, page_rows=32, block=16, max_pages=24, spare=40, per_head=False, e4m3=False, chosen=5, seed=0):
        self.pool = Pool(batch=batch, hkv=len(POLICY), d=D, page_rows=page_rows, max_pages=max_pages, per_head=per_head, e4m3=e4m3, spare=spare, seed=seed)
        self.pool.table.fill_(-1)
        self.blocks = sref.Blocks(self.pool, block)
        self.cfg = sa.make_config(batch=batch, n_q_heads=HQ, n_kv_heads=len(POLICY), head_dim=D, seg_len=SEG, tail_len=TAIL, kv_policy=POLICY, out_fp32=True)
        self.users = torch.zeros(self.pool.n_pages, dtype=I32, device="cuda")
        self.held, self.pos0 = torch.zeros_like(self.pool.rows), torch.zeros(batch, dtype=I64, device="cuda")
        self.granted = torch.zeros(batch, dtype=I32, device="cuda")
        self.n, self.B, self.most = chosen, batch, max_pages * page_rows
        self.pages = self.pool.pages()

    def buffers(self, total, longest):
        n_past = sum(p >> 1 for p in POLICY)
        b = dict(total=total, longest=longest, chosen=torch.full((total, n_past, self.n), -7, dtype=I32, device="cuda"),
                 out=torch.full((total, HQ, D), 77.0, device="cuda"), lse=torch.full((total, HQ), 77.0, device="cuda"),
                 slots=torch.full((total, len(POLICY)), -9, dtype=I64, device="cuda"))
        need = {"reserve": sa.seg_kv_paged_reserve_workspace_bytes(self.cfg, self.pages),
                "choose": sa.seg_kv_paged_choose_workspace_bytes(self.cfg, self.pages, self.blocks.c, total, self.most, self.n),
                "attend": sa.seg_attn_paged_chosen_workspace_bytes(self.cfg, self.pages, self.blocks.c, total, longest, self.most, self.n)}
        b["ws"] = {x: torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for x, n in need.items()}
        return b

    def step(self, b, q, k, v, cu):
        st, ws = torch.cuda.current_stream().cuda_stream, b["ws"]
        rows, total, longest = self.pool.rows, b["total"], b["longest"]
        torch.add(rows, 0, out=self.held)
        sa.seg_kv_paged_reserve(self.cfg, self.pages, self.users, cu, total, longest, rows, self.granted, b["slots"], ws["reserve"],
                                ws["reserve"].numel(), stream=st)
        sa.seg_kv_paged_append(self.cfg, self.pages, None, None, k, v, cu, total, longest, self.pos0, rows, None, rows, st)
        sa.seg_kv_paged_summarize(self.cfg, self.pages, self.blocks.c, self.held, rows, longest, stream=st)
        sa.seg_kv_paged_choose(self.cfg, self.pages, self.blocks.c, q, cu, total, longest, rows, self.most, self.n, 1, 1, b["chosen"], ws["choose"],
                               ws["choose"].numel(), stream=st)
        sa.seg_attn_paged_chosen(self.cfg, self.pages, self.blocks.c, q, cu, total, longest, rows, self.most, b["chosen"], self.n, b["out"], b["lse"],
                                 ws["attend"], ws["attend"].numel(), stream=st)
        sa.seg_kv_paged_release(self.cfg, self.pages, self.users, rows, stream=st)

    def check(self, b, q, sums):
        """The step's results from the pool that it left (released pages are not seen by any of its newest tokens)."""
        rows = self.pool.rows.cpu().tolist()
        lists = sref.chosen(self.pool, self.blocks, q, sums, rows, POLICY, self.n, 1, 1)
        assert torch.equal(b["chosen"].cpu(), lists)
        for t0, m, i in ((sums[i], sums[i + 1] - sums[i], i) for i in range(self.B)):  # the last token of every sequence
            if m:
                cu = [0] * (i + 1) + [1] * (self.B - i)
                t = t0 + m - 1
                want, lse, odd, most_s, most_v = sref.attention(self.pool, q[t:t + 1], cu, rows, POLICY, SEG, TAIL, lists[t:t + 1], self.blocks.rows)
                assert not odd.any()
                delta = D * 2.0 ** -24 * most_s + 2.0 ** -20
                assert ((b["out"][t:t + 1].double().cpu() - want).abs() <= (2 * delta + 2.0 ** -16) * most_v).all()
                assert ((b["lse"][t:t + 1].double().cpu() - lse).abs() <= delta + 2.0 ** -22 * (1 + lse.abs())).all()

    def consistent(self):
        """Every named page has as many users as names, and every other one none."""
        table = self.pool.table.cpu().flatten().long()
        names = torch.bincount(table[table >= 0], minlength=self.pool.n_pages)
        assert torch.equal(names.to(I32), self.users.cpu()) and int(names.max()) <= 1


def _tokens(new, seed):
    g = torch.Generator().manual_seed(seed)
    total = max(1, sum(new))
    q, k, v = (torch.randn((total, h, D), generator=g).to(BF16).cuda() for h in (HQ, len(POLICY), len(POLICY)))
    sums = [sum(new[:i]) for i in range(len(new) + 1)]
    return q, k, v, sums


@pytest.mark.parametrize("kind", [dict(), dict(per_head=True), dict(per_head=True, e4m3=True, page_rows=48, block=48)], ids=["shared", "per_head", "e4m3"])
def test_prompts_steps_eviction_and_release(kind):
    p = Program(3, **kind)
    for i, new in enumerate([[150, 0, 37], [1, 1, 1], [1, 60, 1], [1, 1, 0], [33, 1, 1]]):
        q, k, v, sums = _tokens(new, i)
        b = p.buffers(max(1, sums[-1]), max(new))
        p.step(b, q, k, v, torch.tensor(sums, dtype=I32, device="cuda"))
        assert p.granted.tolist() == [1, 1, 1] and (b["slots"] >= 0).all()
        # rows lie where the reservation said they would
        for t, s in ((sums[x + 1] - 1, x) for x in range(3) if new[x]):
            for h in range(3):
                page, hh, r = p.pool.place(s, h, [int(p.pool.rows[s, h]) - 1])
                assert int(b["slots"][t, h]) == (int(page) * p.pool.heads + hh) * p.pool.R + int(r)
        p.check(b, q, sums)
        p.consistent()
        p.pos0 += torch.tensor(new, device="cuda")
    # back to a budget: rows move, all bounds are formed anew
    cfg, pages, st = p.cfg, p.pages, torch.cuda.current_stream().cuda_stream
    need = sa.seg_kv_paged_evict_workspace_bytes(cfg, pages, p.most, 50)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    sa.seg_kv_paged_evict(cfg, pages, p.pool.rows, p.most, 50, 8, 2, p.pool.rows, ws, need, stream=st)
    sa.seg_kv_paged_release(cfg, pages, p.users, p.pool.rows, stream=st)
    sa.seg_kv_paged_summarize(cfg, pages, p.blocks.c, None, p.pool.rows, p.most, stream=st)
    p.consistent()
    assert p.pool.rows[:, 0].tolist() == [50, 50, 37 + 1 + 1 + 0 + 1]
    new = [1, 2, 20]
    q, k, v, sums = _tokens(new, 9)
    b = p.buffers(sums[-1], max(new))
    p.step(b, q, k, v, torch.tensor(sums, dtype=I32, device="cuda"))
    p.check(b, q, sums)
    p.consistent()
    # the second sequence ends, another one takes its place
    p.pool.rows[1] = 0
    sa.seg_kv_paged_release(cfg, pages, p.users, p.pool.rows, stream=st)
    assert (p.pool.table[1] == -1).all()
    new = [1, 90, 1]
    q, k, v, sums = _tokens(new, 10)
    b = p.buffers(sums[-1], max(new))
    p.step(b, q, k, v, torch.tensor(sums, dtype=I32, device="cuda"))
    p.check(b, q, sums)
    p.consistent()


def _state(p, b):
    return {**p.pool.state(), "table": p.pool.table, "users": p.users, "bounds": p.blocks.bounds, "scale": p.blocks.scale, "granted": p.granted,
            **{x: b[x] for x in ("chosen", "out", "lse", "slots")}}


@pytest.mark.parametrize("new", [[1, 1, 1], [3, 0, 2]], ids=["one_each", "ragged"])
@pytest.mark.parametrize("small", [True, False], ids=["few_blocks", "many_blocks"])
def test_a_captured_step_replays_while_the_cache_grows(new, small):
    """Every replay against the same calls made one by one, with other work and synchronizations between; room for more tokens than there are."""
    kind = dict(page_rows=32, block=16, max_pages=24) if small else dict(page_rows=64, block=16, max_pages=80)
    total = sum(new) + (2 if 0 in new else 0)
    runs = []
    for _ in range(2):
        p = Program(3, **kind)
        q, k, v, sums = _tokens([150, 20, 4000 // 64 if small else 4700], 1)
        b = p.buffers(sums[-1], max(150, sums[-1] - 170))
        p.step(b, q, k, v, torch.tensor(sums, dtype=I32, device="cuda"))
        runs.append((p, p.buffers(total, max(new))))
    inputs = [torch.empty((total, h, D), dtype=BF16, device="cuda") for h in (HQ, 3, 3)]
    cu = torch.zeros(4, dtype=I32, device="cuda")
    cu = None if new == [1, 1, 1] else cu
    if cu is not None:
        cu.copy_(torch.tensor(_tokens(new, 0)[3], dtype=I32))
    (p, b), (e, eb) = runs
    for x in inputs:
        x.zero_()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.step(b, *inputs, cu)
    for i in range(20):
        for x, y in zip(inputs, _tokens([total, 0, 0], 100 + i)):
            x.copy_(y)
        graph.replay()
        e.step(eb, *inputs, cu)
        if i % 3 == 0:
            torch.cuda.synchronize()
        for (name, got), want in zip(_state(p, b).items(), _state(e, eb).values()):
            assert torch.equal(bits(got), bits(want)), (i, name)


def test_calls_on_two_streams_with_workspaces_of_their_own():
    first = torch.cuda.current_stream()
    runs = []
    for seed in (1, 2):
        p = Program(2, seed=seed)
        runs.append((p, [_tokens(n, 10 * seed + i) for i, n in enumerate([[140, 70], [1, 1], [5, 1]])], torch.cuda.Stream()))
    torch.cuda.synchronize()
    kept = []
    for i in range(3):
        for p, tokens, stream in runs:
            q, k, v, sums = tokens[i]
            b = p.buffers(sums[-1], max(sums[1], sums[2] - sums[1]))
            cu = torch.tensor(sums, dtype=I32, device="cuda")
            stream.wait_stream(first)
            with torch.cuda.stream(stream):
                p.step(b, q, k, v, cu)
            kept.append((p, b, q, sums, cu))
    torch.cuda.synchronize()
    for p, b, q, sums, _ in kept[-2:]:
        p.check(b, q, sums)
        p.consistent()


def test_a_pool_without_pages_left_grants_nothing_and_changes_nothing():
    p = Program(3, spare=0, max_pages=6)
    p.users.fill_(1)
    p.users[[4, 9]] = 0
    q, k, v, sums = _tokens([40, 60, 20], 1)  # two, two and one pages
    b = p.buffers(sums[-1], 60)
    sa.seg_kv_paged_reserve(p.cfg, p.pages, p.users, torch.tensor(sums, dtype=I32, device="cuda"), sums[-1], 60, p.pool.rows, p.granted, b["slots"],
                            b["ws"]["reserve"], b["ws"]["reserve"].numel())
    assert p.granted.tolist() == [1, 0, 0] and int(p.users.sum()) == p.pool.n_pages
    assert p.pool.table[0, :2].tolist() == [4, 9] and (p.pool.table[1:] == -1).all()
    assert (b["slots"][:40] >= 0).all() and (b["slots"][40:] == -1).all()
