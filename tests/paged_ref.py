"""Plain 64-bit forms of the operators around a paged cache, written from their definitions (include/segattn.h),
row by row, and helpers that build pools for the tests."""
import math

import numpy as np
import torch

import paper_2605_11744_amd as sa

F64 = torch.float64


# ---- pools ---------------------------------------------------------------------------------------
class Pool:
    """A pool on the GPU: pages in any order, everything that no table names filled with NaN."""

    def __init__(self, *, batch, hkv, d, page_rows, max_pages, per_head=False, e4m3=False, token_major=False, mass=True, pos=True,
                 spare=3, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.B, self.H, self.D, self.R, self.max_pages, self.per_head, self.e4m3 = batch, hkv, d, page_rows, max_pages, per_head, e4m3
        self.heads = 1 if per_head else hkv
        used = batch * (hkv if per_head else 1) * max_pages
        self.n_pages = used + spare
        shape = (batch, hkv, max_pages) if per_head else (batch, max_pages)
        self.table = torch.randperm(self.n_pages, generator=g)[:used].view(shape).to(torch.int32).to(device)
        stored = (self.n_pages, page_rows, self.heads, d) if token_major else (self.n_pages, self.heads, page_rows, d)
        nan = torch.full(stored, 0x7F if e4m3 else float("nan"), dtype=torch.uint8 if e4m3 else torch.bfloat16, device=device)
        self.k, self.v = (nan.clone().permute(0, 2, 1, 3) if token_major else nan.clone() for _ in "kv")
        per_row = (self.n_pages, self.heads, page_rows)
        self.k_scale, self.v_scale = (torch.full(per_row, 127, dtype=torch.uint8, device=device) if e4m3 else None for _ in "kv")
        self.mass = torch.full(per_row, float("nan"), device=device) if mass else None
        self.pos = torch.full(per_row, -1, dtype=torch.int32, device=device) if pos else None
        self.rows = torch.zeros((batch, hkv), dtype=torch.int32, device=device)

    def pages(self):
        return sa.make_pages(k=self.k, v=self.v, table=self.table, max_pages=self.max_pages, page_rows=self.R, n_pages=self.n_pages,
                             per_head=self.per_head, e4m3=self.e4m3, page_stride=self.k.stride(0), head_stride=self.k.stride(1),
                             row_stride=self.k.stride(2), k_scale=self.k_scale, v_scale=self.v_scale, mass=self.mass, pos=self.pos)

    def place(self, b, h, rows):
        """(page, head in page, row in page) of the rows; page -1 where the table names none."""
        rows = torch.as_tensor(rows, dtype=torch.int64)
        table = (self.table[b, h] if self.per_head else self.table[b]).cpu().to(torch.int64)
        page = table[rows // self.R]
        page = torch.where((page >= 0) & (page < self.n_pages), page, -1)
        return page, 0 if self.per_head else h, rows % self.R

    def numbers(self, x, scale, at):
        page, h, r = at
        got = x[page.to(x.device), h, r.to(x.device)]
        if self.e4m3:
            return got.view(torch.float8_e4m3fn).to(F64).cpu() * torch.exp2(scale[page.to(x.device), h, r.to(x.device)].to(F64).cpu() - 127)[:, None]
        return got.to(F64).cpu()

    def kv(self, b, h, rows):
        at = self.place(b, h, rows)
        return self.numbers(self.k, self.k_scale, at), self.numbers(self.v, self.v_scale, at)

    def fill(self, lengths, seed=1):
        """Random rows, masses and positions for lengths [B] or [B][Hkv]."""
        g = torch.Generator().manual_seed(seed)
        for b in range(self.B):
            for h in range(self.H):
                n = lengths[b] if isinstance(lengths[b], int) else lengths[b][h]
                self.rows[b, h] = n
                if n == 0:
                    continue
                page, hh, r = self.place(b, h, range(n))
                ok = page >= 0
                page, r = page[ok].cuda(), r[ok].cuda()
                m = int(ok.sum())
                for x, s in ((self.k, self.k_scale), (self.v, self.v_scale)):
                    new = torch.randn((m, self.D), generator=g)
                    x[page, hh, r] = (new.to(torch.float8_e4m3fn).view(torch.uint8) if self.e4m3 else new.to(torch.bfloat16)).cuda()
                    if self.e4m3:
                        s[page, hh, r] = torch.randint(125, 130, (m,), generator=g, dtype=torch.uint8).cuda()
                if self.mass is not None:
                    self.mass[page, hh, r] = torch.rand(m, generator=g).cuda()
                if self.pos is not None:
                    self.pos[page, hh, r] = torch.arange(n, dtype=torch.int32)[ok].cuda()
        return self

    def state(self):
        return {x: getattr(self, x).clone() for x in ("k", "v", "k_scale", "v_scale", "mass", "pos", "rows") if getattr(self, x) is not None}


def bits(x):
    """Contents that compare equal bit by bit (NaN with NaN)."""
    return x.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[x.element_size()]).cpu()


# ---- definitions -----------------------------------------------------------------------------------
def frequencies(d, *, theta, rotary_dim=0, scaling=0, factor=1.0, trained_len=0.0, low=0.0, high=0.0, inv_freq=None, **_):
    n = rotary_dim or d
    if inv_freq is not None:
        return list(inv_freq)
    f = [theta ** (-2.0 * i / n) for i in range(n // 2)]
    if scaling == sa.SEGATTN_ROPE_LINEAR:
        return [x / factor for x in f]
    if scaling == sa.SEGATTN_ROPE_BY_ROTATIONS:
        kept = [(trained_len * x / (2 * math.pi) - low) / (high - low) for x in f]
    elif scaling == sa.SEGATTN_ROPE_BY_INDEX:
        index = [n * math.log(trained_len / (2 * math.pi * r)) / (2 * math.log(theta)) for r in (high, low)]
        a, b = max(0, math.floor(index[0])), min(n - 1, math.ceil(index[1]))
        kept = [1 - (i - a) / max(b - a, 1e-3) for i in range(n // 2)]
    else:
        return f
    kept = [min(1.0, max(0.0, x)) for x in kept]
    return [x * (k + (1 - k) / factor) for x, k in zip(f, kept)]


def turned(x, positions, rope, inverse=False):
    """x [tokens, heads, D] (float64, CPU) turned; and per element the magnitude that rounding errors scale with."""
    d = x.shape[-1]
    n = rope.get("rotary_dim", 0) or d
    mag = rope.get("magnitude", 0.0) or 1.0
    y, size = x.clone(), x.abs().clone()
    for i, f in enumerate(frequencies(d, **rope)):
        a, b = (2 * i, 2 * i + 1) if rope.get("interleaved") else (i, i + n // 2)
        t = torch.as_tensor(positions, dtype=F64) * f * (-1 if inverse else 1)
        c, s = (mag * t.cos())[:, None], (mag * t.sin())[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = mag * (x[..., a].abs() + x[..., b].abs())
    return y, size


def e4m3_rows(x):
    """Bits and scale bytes of rows x [rows, D] (float64): every finite element rounded once, the rest NaN."""
    most = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    e = torch.tensor([0 if m == 0 else max(-119, math.ceil(math.log2(m / 448))) for m in most.tolist()])
    y = x / torch.exp2(e.to(F64))[:, None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    q = (y / step).round() * step  # to nearest even, exactly representable
    q = torch.where(x.isfinite(), q, torch.nan)
    return q.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def first_row(n, policy, seg, tail):
    start = max(0, n - 1) // seg * seg
    return 0 if policy & 2 else max(0, start - tail) if policy & 1 else start


def attention(pool, q, lengths, policy, seg, tail, scale=0.0, max_rows=None):
    """out, lse, weights {(b, h): (rows, summed weights)}, and the largest |scores sum of products| and |v| met."""
    B, hq, d = q.shape
    g = hq // pool.H
    out, lse = torch.zeros((B, hq, d), dtype=F64), torch.full((B, hq), -math.inf, dtype=F64)
    weights, most_s, most_v = {}, 0.0, 0.0
    scale = scale or 1 / math.sqrt(d)
    for b in range(B):
        for h in range(pool.H):
            n = lengths[b] if isinstance(lengths[b], int) else lengths[b][h]
            n = min(n, max_rows) if max_rows else n
            rows = torch.arange(first_row(n, policy[h], seg, tail), n)
            if len(rows):
                rows = rows[pool.place(b, h, rows)[0] >= 0]
            if len(rows) == 0:
                continue
            k, v = pool.kv(b, h, rows)
            qq = q[b, h * g:(h + 1) * g].to(F64).cpu()
            s = qq @ k.T * scale
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
            p = (s - lse[b, h * g:(h + 1) * g, None]).exp()
            out[b, h * g:(h + 1) * g] = p @ v
            weights[b, h] = rows, p.sum(0)
            most_s = max(most_s, float((qq.abs() @ k.abs().T).max()) * scale)
            most_v = max(most_v, float(v.abs().max()))
    return out, lse, weights, most_s, most_v


def evicted(pool, keep, recent, first, policy, max_rows=None):
    """The state that an eviction leaves, from the definition: kept rows by sorting, moves one at a time."""
    s = {x: y.cpu().clone() for x, y in pool.state().items()}
    moved = 0
    for b in range(pool.B):
        for h in range(pool.H):
            n = int(s["rows"][b, h])
            n = min(n, max_rows) if max_rows else n
            if not policy[h] & 2 or n <= keep:
                continue
            page, hh, r = pool.place(b, h, range(n))
            ok = page >= 0
            pos = [int(s["pos"][page[i], hh, r[i]]) if ok[i] else None for i in range(n)]
            newest = max((p for p in pos if p is not None), default=0)
            def key(i):
                if pos[i] > newest - recent:
                    return 2, pos[i]
                if first > 0 and pos[i] < first:
                    return 1, 0.0
                m = float(s["mass"][page[i], hh, r[i]])
                return 0, m if m > 0 else 0.0
            there = [i for i in range(n) if ok[i]]
            order = sorted(sorted(there), key=key, reverse=True)  # (stable: equal keys stay in the order of rows)
            kept = set(order[:sum(i < keep for i in there)])
            places = [i for i in there if i < keep and i not in kept]
            movers = [i for i in there if i >= keep and i in kept]
            assert len(places) == len(movers)
            for to, of in zip(places, movers):
                for x in s:
                    if x != "rows":
                        s[x][page[to], hh, r[to]] = s[x][page[of], hh, r[of]]
                moved += 1
            s["rows"][b, h] = keep
    return s, moved
