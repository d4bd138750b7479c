"""Plain forms of the operators for sparse attention over a paged cache, written from their definitions (include/segattn.h), one
sequence, head and token at a time: whole numbers as Python's, attention in 64 bits."""
import math

import torch

import paged_ref as ref

F64 = torch.float64


# ---- tables ----------------------------------------------------------------------------------------
def reserved(*, table, users, rows, new, page_rows, per_head, policy, seg, tail, newest=False, slots=None, cu=None):
    """table, users, granted, slots after a reservation; rows [B][Hkv], new [B] as lists, the rest CPU tensors."""
    table, users = table.clone(), users.clone()
    B, H, n_pages, max_pages = len(rows), len(rows[0]), len(users), table.shape[-1]
    free = [p for p in range(n_pages) if users[p] <= 0]
    granted, asked, given = [], 0, 0
    for b in range(B):
        wanted, fits = [], True
        for h in range(H):
            held = min(max(0, rows[b][h]), max_pages * page_rows)
            end = held + new[b]
            fits &= end <= max_pages * page_rows or new[b] == 0
            lo = max(held, ref.first_row(end, policy[h], seg, tail)) if newest else held
            if new[b]:
                wanted += [(h if per_head else 0, r // page_rows) for r in range(lo, end)]
        named = lambda h, e: 0 <= int(table[b, h, e] if per_head else table[b, e]) < n_pages
        missing = [x for x in sorted(set(wanted)) if not named(*x)] if fits else []
        asked += len(missing)
        ok = fits and (not missing or asked <= len(free))
        granted.append(int(ok))
        if ok:
            for h, e in missing:
                page = free[given]
                given += 1
                users[page] = 1
                if per_head:
                    table[b, h, e] = page
                else:
                    table[b, e] = page
    if slots is not None:
        slots = slots.clone()
        for b in range(B):
            for i in range(new[b]):
                for h in range(H):
                    r = min(max(0, rows[b][h]), max_pages * page_rows) + i
                    page = -1
                    if granted[b] and r < max_pages * page_rows:
                        page = int(table[b, h, r // page_rows] if per_head else table[b, r // page_rows])
                    place = page * page_rows + r % page_rows if per_head else (page * H + h) * page_rows + r % page_rows
                    slots[cu[b] + i, h] = place if 0 <= page < n_pages else -1
    return table, users, granted, slots


def released(*, table, users, rows, page_rows, per_head, policy, seg, tail):
    table, users = table.clone(), users.clone()
    B, H, n_pages, max_pages = len(rows), len(rows[0]), len(users), table.shape[-1]
    for b in range(B):
        for h in range(H if per_head else 1):
            kept = set()
            for k in ([h] if per_head else range(H)):
                n = min(max(0, rows[b][k]), max_pages * page_rows)
                kept |= {r // page_rows for r in range(ref.first_row(n, policy[k], seg, tail), n)}
            line = table[b, h] if per_head else table[b]
            for e in range(max_pages):
                if e not in kept and 0 <= int(line[e]) < n_pages:
                    users[int(line[e])] -= 1
                    line[e] = -1
    return table, users


# ---- bounds ----------------------------------------------------------------------------------------
def least_exponent(most, least=None):
    """Smallest e with most <= 127 * 2^e, exactly."""
    if most == 0:
        return least
    e = math.frexp(most)[1] - 8
    while most > 127 * 2.0 ** e:
        e += 1
    return e if least is None else max(e, least)


def bounds_of(keys):
    """keys [rows, D] (float64): upper and lower bounds (whole numbers) and the scale byte."""
    keys = torch.where(keys.isfinite() & (keys.abs() <= float(torch.finfo(torch.float32).max)), keys, 0.0)
    e = least_exponent(float(keys.abs().max()), -80)
    return torch.ceil(keys.amax(0) * 2.0 ** -e), torch.floor(keys.amin(0) * 2.0 ** -e), e + 127


class Blocks:
    """Storage for the bounds of a pool's blocks, filled with values that no result may depend on."""

    def __init__(self, pool, block_rows, device="cuda"):
        import paper_2605_11744_amd as sa
        shape = (pool.n_pages, pool.heads, pool.R // block_rows)
        self.rows = block_rows
        self.bounds = torch.full(shape + (2, pool.D), 99, dtype=torch.int8, device=device)
        self.scale = torch.full(shape, 200, dtype=torch.uint8, device=device)
        self.c = sa.make_blocks(block_rows=block_rows, bounds=self.bounds, scale=self.scale)

    def at(self, pool, b, h, j):
        """Place of block j of (b, h), or None without a page."""
        (page,), hh, (r,) = pool.place(b, h, [j * self.rows])
        return None if page < 0 else (int(page), hh, int(r) // self.rows)


def summarized(pool, blocks, rows_from, rows, policy, max_new):
    """bounds and scale after the call; rows_from, rows [B][Hkv] lists."""
    bounds, scale = blocks.bounds.cpu().clone(), blocks.scale.cpu().clone()
    for b in range(pool.B):
        for h in range(pool.H):
            if not policy[h] & 2:
                continue
            first = rows_from[b][h] // blocks.rows
            for j in range(first, min(rows[b][h] // blocks.rows, first + -(-max_new // blocks.rows))):
                at = blocks.at(pool, b, h, j)
                if at is None:
                    continue
                hi, lo, byte = bounds_of(pool.kv(b, h, range(j * blocks.rows, (j + 1) * blocks.rows))[0])
                bounds[at][0], bounds[at][1], scale[at] = hi.to(torch.int8), lo.to(torch.int8), byte
    return bounds, scale


# ---- choice ----------------------------------------------------------------------------------------
def chosen(pool, blocks, q, cu, rows, policy, n_chosen, first, recent, max_rows=None, fill=-7):
    """chosen [total, n_past, n_chosen]; rows [B][Hkv] list, q [total, Hq, D]."""
    past = [h for h in range(pool.H) if policy[h] & 2]
    bounds, scale = blocks.bounds.cpu().to(torch.int64), blocks.scale.cpu()
    out = torch.full((q.shape[0], len(past), n_chosen), fill, dtype=torch.int32)
    g = q.shape[1] // pool.H
    for b in range(pool.B):
        m = cu[b + 1] - cu[b]
        for i in range(m):
            for x, h in enumerate(past):
                end = rows[b][h] - m + i + 1
                end = max(0, min(end, max_rows) if max_rows else end)
                own = (end - 1) // blocks.rows if end else -1
                if own + 1 <= n_chosen:
                    got = list(range(own + 1))
                else:
                    group = q[cu[b] + i, h * g:(h + 1) * g].to(F64).cpu()
                    group = torch.where(group.isfinite(), group, 0.0)
                    most = float(group.abs().max())
                    q8 = (group * 2.0 ** -least_exponent(most) if most else group).round().to(torch.int64)  # half to even
                    score = []
                    for j in range(first, own - recent + 1):
                        at = blocks.at(pool, b, h, j)
                        if at is None:
                            score.append((-math.inf, -j))
                            continue
                        dot = torch.where(q8 > 0, q8 * bounds[at][0], q8 * bounds[at][1]).sum(-1).max()
                        score.append((int(dot) * 2.0 ** (int(scale[at]) - 127), -j))
                    got = sorted([*range(first), *(-j for _, j in sorted(score, reverse=True)[:n_chosen - first - recent]),
                                  *range(own - recent + 1, own + 1)])
                out[cu[b] + i, x] = torch.tensor(got + [-1] * (n_chosen - len(got)), dtype=torch.int32)
    return out


# ---- attention -------------------------------------------------------------------------------------
def attention(pool, q, cu, rows, policy, seg, tail, lists, block_rows, scale=0.0, max_rows=None):
    """out, lse, whether a query head sees a value that is not finite, and the largest |scores' sum of products| and |v| met.  Tokens
    behind the last sequence: NaN."""
    total, hq, d = q.shape
    g = hq // pool.H
    out, lse = torch.full((total, hq, d), math.nan, dtype=F64), torch.full((total, hq), math.nan, dtype=F64)
    scale = scale or 1 / math.sqrt(d)
    past = [h for h in range(pool.H) if policy[h] & 2]
    most_s, most_v = 0.0, 0.0
    odd = torch.zeros((total, hq), dtype=torch.bool)
    for b in range(pool.B):
        m = cu[b + 1] - cu[b]
        for h in range(pool.H):
            n = rows[b][h]
            at = torch.arange(max(n, 0))
            if len(at):
                ok = pool.place(b, h, at)[0] >= 0
                kk, vv = pool.kv(b, h, at)
            for i in range(m):
                t = cu[b] + i
                heads = slice(h * g, (h + 1) * g)
                end = n - m + i + 1
                end = max(0, min(end, max_rows) if max_rows else end)
                if policy[h] & 2:
                    mine = lists[t, past.index(h)].to(torch.int64)
                    see = (mine[mine >= 0][:, None] * block_rows + torch.arange(block_rows)).flatten()
                    see = see[see < end]
                else:
                    see = torch.arange(ref.first_row(end, policy[h], seg, tail), end)
                see = see[ok[see]] if len(see) else see
                out[t, heads], lse[t, heads] = 0.0, -math.inf
                if not len(see):
                    continue
                k, v = kk[see], vv[see]
                odd[t, heads] = not bool(k.isfinite().all() and v.isfinite().all())
                qq = q[t, heads].to(F64).cpu()
                s = qq @ k.T * scale
                z = torch.logsumexp(s, -1)
                lse[t, heads], out[t, heads] = z, (s - z[:, None]).exp() @ v
                if not odd[t, heads].any():
                    most_s = max(most_s, float((qq.abs() @ k.abs().T).max()) * scale)
                    most_v = max(most_v, float(v.abs().max()))
    return out, lse, odd, most_s, most_v
