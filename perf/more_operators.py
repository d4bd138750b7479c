"""Performance cases of libsegattn's operators for sparse attention over a paged cache: what a serving program
calls beside appending rows, so that its tables are kept on the GPU and a token reads a few blocks of its history.

    reserve    seg_kv_paged_reserve: pages for the tokens that are about to be appended, taken from those that no
               table names, and the place of every new row
    release    seg_kv_paged_release: pages whose rows no head sees any more, or of sequences that ended, given back
    summarize  seg_kv_paged_summarize: upper and lower bounds of the keys of every block that became complete, in 8 bits
    choose     seg_kv_paged_choose: for every token and long-range KV head the blocks whose bounds promise the
               highest scores, the first and the newest ones always
    attend     seg_attn_paged_chosen: attention of new tokens over the rows of those blocks, and of the other
               heads over their windows

`policy` has a digit per KV head: 0 own segment only, 1 carried tail, 2 past, 3 tail and past.  A sequence holds
`held` rows before its `new` tokens.  Values are N(0, 1) rounded to bf16, as in every workload of this repository.
"""
import math

import torch

own = False

BF16, F32, F64, I32, I64, U8, I8 = (torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8, torch.int8)
E4M3 = torch.float8_e4m3fn

# Exponent of a block's smallest scale, and the keys' range that the scale covers.
LEAST_EXPONENT, MOST = -80, 127


def listed():
    return [
        # Pages for a generation step of 48 sequences: one of 64 opens a new page.
        {"name": "reserve_step", "op": "reserve", "batch": 48, "held_lo": 500, "held_hi": 9000, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": False, "seg": 4096, "tail": 1024, "policy": "22222222", "newest": False,
         "short": False},
        # Prompts of 1K to 32K handed over after their prefill, pages per head, only the rows that will still be seen; the
        # pool is too small for all of them.
        {"name": "reserve_prompts", "op": "reserve", "batch": 24, "held_lo": 0, "held_hi": 0, "new_lo": 1000, "new_hi": 32768,
         "hq": 32, "hkv": 8, "d": 128, "page": 32, "per_head": True, "seg": 4096, "tail": 1024, "policy": "33111111",
         "newest": True, "short": True},
        # Requests that ended among others that go on, small shared pages.
        {"name": "release_ended", "op": "release", "batch": 96, "held_lo": 10, "held_hi": 20000, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 16, "per_head": False, "seg": 4096, "tail": 1024, "policy": "22222222", "ended": 3},
        # A server's step under segmented execution: pages behind the windows of the short-range heads.
        {"name": "release_windows", "op": "release", "batch": 64, "held_lo": 4097, "held_hi": 65536, "new_lo": 1, "new_hi": 1,
         "hq": 32, "hkv": 8, "d": 128, "page": 64, "per_head": True, "seg": 4096, "tail": 1024, "policy": "33111111", "ended": 0},
        # A generation step: few of the sequences complete a block.
        {"name": "summarize_step", "op": "summarize", "batch": 64, "held_lo": 100, "held_hi": 4000, "new_lo": 1, "new_hi": 1,
         "hq": 32, "hkv": 8, "d": 128, "page": 64, "per_head": False, "e4m3": False, "seg": 4096, "tail": 1024,
         "policy": "22222222", "block": 16},
        # Prompts of different lengths that an 8-bit cache has taken.
        {"name": "summarize_prompts", "op": "summarize", "batch": 9, "held_lo": 0, "held_hi": 900, "new_lo": 61, "new_hi": 32768,
         "hq": 32, "hkv": 8, "d": 128, "page": 128, "per_head": False, "e4m3": True, "seg": 4096, "tail": 1024,
         "policy": "22222222", "block": 64},
        # One user's generation behind 128K tokens.
        {"name": "choose_one", "op": "choose", "batch": 1, "held_lo": 131071, "held_hi": 131071, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": False, "seg": 4096, "tail": 1024, "policy": "22222222", "block": 64,
         "chosen": 64, "first": 1, "recent": 2},
        # A server's step: contexts of 4K to 64K, 2K rows of each.
        {"name": "choose_step", "op": "choose", "batch": 64, "held_lo": 4097, "held_hi": 65536, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": False, "seg": 4096, "tail": 1024, "policy": "22222222", "block": 64,
         "chosen": 32, "first": 1, "recent": 2},
        # Chunks of prompts behind what is there already: every token has its own choice.
        {"name": "choose_chunk", "op": "choose", "batch": 3, "held_lo": 2500, "held_hi": 60000, "new_lo": 1, "new_hi": 2048, "hq": 32,
         "hkv": 8, "d": 128, "page": 128, "per_head": False, "seg": 4096, "tail": 1024, "policy": "33331111", "block": 64,
         "chosen": 32, "first": 1, "recent": 2},
        # One user's generation: 4K of 128K rows.
        {"name": "attend_one", "op": "attend", "batch": 1, "held_lo": 131071, "held_hi": 131071, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": False, "e4m3": False, "seg": 4096, "tail": 1024, "policy": "22222222",
         "block": 64, "chosen": 64, "first": 1, "recent": 2, "f32": False},
        # A server's step under segmented execution: an 8-bit cache, a quarter of the heads long-range.
        {"name": "attend_step", "op": "attend", "batch": 48, "held_lo": 4097, "held_hi": 65536, "new_lo": 1, "new_hi": 1, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": True, "e4m3": True, "seg": 4096, "tail": 1024, "policy": "33111111",
         "block": 64, "chosen": 32, "first": 1, "recent": 2, "f32": False},
        # Chunks of prompts, half of the heads long-range: the largest call.
        {"name": "attend_chunk", "op": "attend", "batch": 3, "held_lo": 2500, "held_hi": 60000, "new_lo": 1, "new_hi": 2048, "hq": 32,
         "hkv": 8, "d": 128, "page": 128, "per_head": False, "e4m3": False, "seg": 4096, "tail": 1024, "policy": "33331111",
         "block": 64, "chosen": 32, "first": 1, "recent": 2, "f32": False},
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (16, 4, 128), (8, 8, 128), (16, 2, 128), (4, 4, 64), (16, 4, 64), (32, 8, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["reserve", "release", "summarize", "choose", "choose", "attend", "attend", "attend"])
    hq, hkv, d = rng.choice(HEADS)
    past = rng.choice([hkv, hkv, max(1, hkv // 4), max(1, hkv // 2)])
    c = {"op": op, "hq": hq, "hkv": hkv, "d": d, "seg": rng.choice([512, 1000, 4096]), "tail": rng.choice([0, 128, 512]),
         "policy": rng.choice("23") * past + "1" * (hkv - past), "per_head": rng.random() < 0.4}
    block = rng.choice([16, 32, 48, 64, 64, 128])
    step = rng.random() < 0.5
    held = _log_int(rng, 20, 60000)
    new = 1 if step else _log_int(rng, 2, 1200)
    rows = held + new
    c.update(held_lo=held // rng.choice([1, 2, 5]), held_hi=held, new_lo=1 if step else rng.randint(0, new // 2), new_hi=new)
    if op in ("reserve", "release"):
        c.update(batch=_log_int(rng, 1, max(2, min(100, 1500000 // rows))), page=rng.choice([16, 24, 32, 64, 128]))
        if op == "reserve":
            c.update(newest=rng.random() < 0.5, short=rng.random() < 0.3)
        else:
            c.update(ended=rng.choice([0, 2, 5]))
        return c
    c.update(block=block, page=block * rng.choice([1, 1, 2, 4]))
    if op == "summarize":
        c.update(batch=_log_int(rng, 1, max(2, min(64, 400000 // rows))), e4m3=rng.random() < 0.4)
        return c
    c.update(batch=_log_int(rng, 1, max(2, min(64, 1500000 // rows))) if step else rng.randint(1, 2), chosen=rng.randint(4, 64),
             first=rng.choice([0, 1]), recent=rng.choice([1, 2, 3]))
    if op == "attend":
        c.update(chosen=min(c["chosen"], max(4, 2048 // block)) if not step else c["chosen"], e4m3=rng.random() < 0.4,
                 f32=rng.random() < 0.3)
    return c


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths spread over lo..hi: both ends, then multiples of the golden ratio."""
    return [lo if i == 0 else hi if i == 1 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _sizes(case):
    """Rows held before the new tokens, and new tokens, of every sequence."""
    B = case["batch"]
    return _spread(B, case["held_lo"], case["held_hi"]), _spread(B, case["new_lo"], case["new_hi"])


def _policy(case):
    return [int(x) for x in case["policy"]]


def _past(case):
    return [h for h, p in enumerate(_policy(case)) if p & 2]


def _window(case, p, row):
    """First row that a head of policy p sees from the token at `row`."""
    start = max(0, row) // case["seg"] * case["seg"]
    return 0 if p & 2 else max(0, start - case["tail"]) if p & 1 else start


def _tables(case, g, lo, hi, spare, most):
    """A table that names pages in any order for rows lo..hi of every head, and how many tables name each page."""
    B, H, R = case["batch"], case["hkv"], case["page"]
    lo, hi = torch.tensor(lo, dtype=I64), torch.tensor(hi, dtype=I64)
    if not case["per_head"]:
        lo, hi = lo.min(dim=1, keepdim=True).values, hi.max(dim=1, keepdim=True).values
    at = torch.arange(most)
    held = ((at >= (lo // R)[..., None]) & (at < (-(-hi // R))[..., None])).cuda()
    used = int(held.sum())
    pages = torch.randperm(used + spare, generator=g, device="cuda")[:used]
    table = torch.full(held.shape, -1, dtype=I32, device="cuda")
    table[held] = pages.to(I32)
    users = torch.zeros(used + spare, dtype=I32, device="cuda")
    users[pages] = 1
    return table if case["per_head"] else table[:, 0].contiguous(), users


def _normal(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=BF16)


def _pool(case, s, g, n, filled):
    heads = 1 if case["per_head"] else case["hkv"]
    shape = (n, heads, case["page"], case["d"])
    if filled:
        s["k"], s["v"] = _normal(g, shape), _normal(g, shape)
    else:  # no operator of the case reads it
        s["k"], s["v"] = torch.empty(shape, dtype=BF16, device="cuda"), torch.empty(shape, dtype=BF16, device="cuda")
    if case.get("e4m3"):
        s["k"], s["v"] = s["k"].to(E4M3).view(U8), s["v"].to(E4M3).view(U8)
        s["k_scale"], s["v_scale"] = (torch.randint(125, 129, shape[:3], generator=g, device="cuda", dtype=U8) for _ in "kv")
    if "block" in case:
        blocks = (n, heads, case["page"] // case["block"])
        s["bounds"] = torch.zeros(blocks + (2, case["d"]), dtype=I8, device="cuda")
        s["scale"] = torch.zeros(blocks, dtype=U8, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, B, hq, hkv, d, R = case["op"], case["batch"], case["hq"], case["hkv"], case["d"], case["page"]
    held, new = _sizes(case)
    both = [a + b for a, b in zip(held, new)]
    most = max(1, max(-(-n // R) for n in both))
    s = {"case": case, "most": most, "total": sum(new), "longest": max(1, max(new)), "max_rows": max(1, max(both))}
    cu = [sum(new[:i]) for i in range(B + 1)]
    s["cu"] = torch.tensor(cu, dtype=I32, device="cuda")
    s["held"] = torch.tensor(held, dtype=I32, device="cuda")[:, None].expand(B, hkv).contiguous()
    s["rows"] = torch.tensor(both, dtype=I32, device="cuda")[:, None].expand(B, hkv).contiguous()
    if op in ("reserve", "release"):
        if op == "reserve":
            lo = [[_window(case, p, n - 1) for p in _policy(case)] for n in held]
            per_head = hkv if case["per_head"] else 1
            need = sum(-(-z // R) - -(-a // R) for a, z in zip(held, both)) * per_head
            if case["newest"] and case["per_head"]:
                need = sum(-(-z // R) - max(-(-a // R), _window(case, p, z - 1) // R) for a, z in zip(held, both) for p in _policy(case))
            table, users = _tables(case, g, lo, [[n] * hkv for n in held], max(1, need * 2), most)
            free = (users == 0).nonzero()[:, 0]  # other programs' pages among them
            keep = max(1, int(need * 0.6)) if case["short"] else need + 3
            users[free[torch.randperm(len(free), generator=g, device="cuda")[keep:]]] = 1
            s["slots"] = torch.empty((s["total"], hkv), dtype=I64, device="cuda")
        else:
            # what the step before had to see: a segment's windows began up to a segment earlier
            lo = [[_window(case, p, n - 1 - case["seg"]) for p in _policy(case)] for n in both]
            table, users = _tables(case, g, lo, [[n] * hkv for n in both], 7, most)
            shared = torch.rand(users.shape, generator=g, device="cuda") < 0.05
            users += (shared & (users > 0)).to(I32)
            if case["ended"]:
                s["rows"][::case["ended"]] = 0
        n, t = users.numel(), table.numel()
        s["kept0"] = torch.cat([users, table.flatten(), torch.zeros(B, dtype=I32, device="cuda")])
        s["kept"] = s["kept0"].clone()
        s["users"], s["table"], s["granted"] = s["kept"][:n], s["kept"][n:n + t].view(table.shape), s["kept"][n + t:]
        _pool(case, s, g, n, False)
        return s
    lo = [[_window(case, p, n) for p in _policy(case)] for n in held]
    s["table"], users = _tables(case, g, lo, [[n] * hkv for n in both], 3, most)
    _pool(case, s, g, users.numel(), op != "choose")
    if op == "summarize":
        return s
    past, br = _past(case), case["block"]
    s["past"] = torch.tensor(past, device="cuda")
    s["q"] = _normal(g, (s["total"], hq, d))
    if op == "choose":
        # The largest and the smallest of a block's normal values in a channel, in the steps of two scales.
        e = torch.randint(0, 2, s["scale"].shape, generator=g, device="cuda")
        size = torch.exp2(5.0 - e.to(F32))[..., None, None]
        x = (2.4 + 0.43 * torch.randn(s["bounds"].shape, generator=g, device="cuda")) * size
        x[..., 1, :] *= -1
        s["bounds"] = x.round().clamp(-MOST, MOST).to(I8)
        s["scale"] = (122 + e).to(U8)
        s["chosen"] = torch.empty((s["total"], len(past), case["chosen"]), dtype=I32, device="cuda")
        return s
    # lists as the choice leaves them: the first and the newest blocks, others at random, in order
    s["chosen"] = torch.full((s["total"], len(past), case["chosen"]), -1, dtype=I32, device="cuda")
    for b in range(B):
        own_block = (held[b] + torch.arange(new[b], device="cuda")) // br
        for i in range(0, new[b], 512):
            o = own_block[i:i + 512, None, None]
            at = torch.arange(both[b] // br + 1, device="cuda")
            x = torch.rand((len(o), len(past), len(at)), generator=g, device="cuda")
            x = x.masked_fill((at < case["first"]) | (at > o - case["recent"]), 2.0).masked_fill(at > o, -1.0)
            x, idx = x.sort(dim=-1, descending=True)
            n = min(case["chosen"], len(at))
            idx = torch.where(x[..., :n] >= 0, idx[..., :n], 1 << 30).sort(dim=-1).values
            s["chosen"][cu[b] + i:cu[b] + i + len(o), :, :n] = torch.where(idx < 1 << 30, idx, -1).to(I32)
    s["out"] = torch.empty((s["total"], hq, d), dtype=F32 if case["f32"] else BF16, device="cuda")
    s["lse"] = torch.empty((s["total"], hq), dtype=F32, device="cuda")
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------------
def _starts(case, rows):
    """First visible row of every head, [B, hkv], from the newest of rows [B, hkv]."""
    p = torch.tensor(_policy(case), device="cuda")
    start = (rows - 1).clamp(min=0) // case["seg"] * case["seg"]
    carried = torch.where(p & 1 > 0, case["tail"], 0)
    return torch.where(p & 2 > 0, 0, (start - carried).clamp(min=0))


def _named(s):
    return (s["table"] >= 0) & (s["table"] < s["k"].shape[0])


def _tokens(s):
    """Sequence of every new token, and its number there."""
    t = torch.arange(s["total"], device="cuda")
    b = torch.searchsorted(s["cu"].to(I64), t, right=True) - 1
    return b, t - s["cu"][b]


def _run_reserve(s):
    case = s["case"]
    R, H = case["page"], case["hkv"]
    new = (s["cu"][1:] - s["cu"][:-1]).to(I64)
    rows = s["held"].to(I64)
    end = rows + new[:, None]
    fits = (end <= s["most"] * R).all(1)
    lo = torch.maximum(rows, _starts(case, end)) if case["newest"] else rows
    at = torch.arange(s["most"], device="cuda")
    wanted = (at >= (lo // R)[..., None]) & (at < (-(-end // R))[..., None]) & ((new > 0) & fits)[:, None, None]
    wanted = wanted if case["per_head"] else wanted.any(1)
    missing = wanted & ~_named(s)
    need = missing.flatten(1).sum(1)
    free = (s["users"] <= 0).nonzero()[:, 0]
    granted = fits & ((need.cumsum(0) <= free.numel()) | (need == 0))
    take = missing & granted.view((-1,) + (1,) * (missing.dim() - 1))
    pages = free[:int(take.sum())]
    s["table"][take] = pages.to(I32)
    s["users"][pages] = 1
    s["granted"].copy_(granted)
    b, i = _tokens(s)
    row = rows[b] + i[:, None]
    head = torch.arange(H, device="cuda")
    if case["per_head"]:
        page, place = s["table"][b[:, None], head, row // R].to(I64), row % R
    else:
        page = s["table"][b[:, None], row // R].to(I64)
        place = head * R + row % R
    slots = torch.where((page >= 0) & granted[b][:, None], page * (R if case["per_head"] else R * H) + place, -1)
    return {"users": s["users"], "table": s["table"], "granted": s["granted"], "slots": slots}


def _run_release(s):
    case = s["case"]
    R, rows = case["page"], s["rows"].to(I64)
    at = torch.arange(s["most"], device="cuda")
    keep = (at >= (_starts(case, rows) // R)[..., None]) & (at < (-(-rows // R))[..., None])
    keep = keep if case["per_head"] else keep.any(1)
    drop = _named(s) & ~keep
    s["users"] -= torch.bincount(s["table"][drop].to(I64), minlength=s["users"].numel()).to(I32)
    s["table"][drop] = -1
    return {"users": s["users"], "table": s["table"]}


def _take(s, name, slot, dtype=F32):
    """The rows `slot` names, as numbers of `dtype`."""
    x = s[name].reshape(-1, s["case"]["d"])[slot]
    if not s["case"]["e4m3"]:
        return x.to(dtype)
    return torch.ldexp(x.view(E4M3).to(dtype), (s[name + "_scale"].reshape(-1)[slot].to(I32) - 127)[..., None])


def _slot(s, b, h, row):
    """Place of rows of heads h of sequences b among all rows of the pool's heads, and whether they have one."""
    case = s["case"]
    R, at = case["page"], (row // case["page"]).clamp(0, s["most"] - 1)
    page = (s["table"][b, h, at] if case["per_head"] else s["table"][b, at]).to(I64)
    slot = page * R + row % R if case["per_head"] else (page * case["hkv"] + h) * R + row % R
    return slot.clamp(min=0), (page >= 0) & (row >= 0)


def _run_summarize(s):
    case = s["case"]
    br, past = case["block"], torch.tensor(_past(case), device="cuda")
    first, n = s["held"][:, past].to(I64) // br, s["rows"][:, past].to(I64) // br
    at = torch.arange(s["longest"] // br + 2, device="cuda") + first[..., None]
    b, h, i = (at < n[..., None]).nonzero(as_tuple=True)
    block, h = at[b, h, i], past[h]
    for j in range(0, len(b), 8192):
        bb, hh, blk = b[j:j + 8192], h[j:j + 8192], block[j:j + 8192]
        slot, _ = _slot(s, bb[:, None], hh[:, None], blk[:, None] * br + torch.arange(br, device="cuda"))
        x = _take(s, "k", slot)
        hi, lo = x.amax(1), x.amin(1)
        m, e = torch.frexp(torch.maximum(hi.abs(), lo.abs()).amax(-1))
        e = torch.where(m == 0, LEAST_EXPONENT, e - 7 + (m > MOST / 128).to(I32)).clamp(min=LEAST_EXPONENT)
        to = slot[:, 0] // br
        s["bounds"].view(-1, 2, case["d"])[to] = torch.stack([torch.ldexp(hi, -e[:, None]).ceil(), torch.ldexp(lo, -e[:, None]).floor()], 1).to(I8)
        s["scale"].view(-1)[to] = (e + 127).to(U8)
    return {"bounds": s["bounds"], "scale": s["scale"]}


def _run_choose(s):
    case = s["case"]
    br, n, hkv, d = case["block"], case["chosen"], case["hkv"], case["d"]
    past, g = s["past"], case["hq"] // case["hkv"]
    b_of, i_of = _tokens(s)
    row = s["rows"][b_of][:, past].to(I64) - (s["cu"][b_of + 1] - s["cu"][b_of])[:, None] + i_of[:, None]  # [tokens, past heads]
    q = s["q"].view(-1, hkv, g, d)[:, past].to(F32)
    m, e = torch.frexp(q.abs().amax((-1, -2)))
    q = torch.ldexp(q, (7 - e - (m > MOST / 128).to(I32))[..., None, None]).round()
    q = torch.cat([q.clamp(min=0), q.clamp(max=0)], -1)  # with the upper bounds, and with the lower ones
    at = torch.arange(-(-s["max_rows"] // br), device="cuda")
    chosen = torch.full((s["total"], len(past), n), -1, dtype=I32, device="cuda")
    if s["longest"] == 1 and s["total"] == case["batch"]:  # every token has blocks of its own
        some = max(1, (1 << 17) // len(at))
        parts = [(slice(t, t + some), slice(t, t + some)) for t in range(0, s["total"], some)]
    else:  # a sequence's tokens share its blocks
        new = _sizes(case)[1]
        parts = [(slice(b, b + 1), slice(sum(new[:b]) + t, sum(new[:b]) + min(t + 256, m)))
                 for b, m in enumerate(new) for t in range(0, m, 256)]
    for sequences, tokens in parts:
        bb = torch.arange(case["batch"], device="cuda")[sequences]
        slot, ok = _slot(s, bb[:, None, None], past[:, None], at * br)
        k = s["bounds"].view(-1, 2 * d)[slot // br].to(F32)  # [sequences, past heads, blocks, 2 d]
        size = torch.exp2(s["scale"].view(-1)[slot // br].to(F32) - 127)
        x = q[tokens].view(len(bb), -1, len(past), g, 2 * d).transpose(1, 2).flatten(2, 3)
        x = x @ k.transpose(-1, -2)  # whole numbers below 2^24: exact
        x = x.view(len(bb), len(past), -1, g, len(at)).amax(3) * size[:, :, None]
        x = x.masked_fill(~ok[:, :, None], -3e38).transpose(1, 2).flatten(0, 1)  # [tokens, past heads, blocks]
        o = (row[tokens] // br)[..., None]
        x = x.masked_fill((at < case["first"]) | (at > o - case["recent"]), math.inf).masked_fill(at > o, -math.inf)
        idx = x.sort(dim=-1, descending=True, stable=True).indices[..., :n]
        idx = torch.where(idx <= o, idx, 1 << 30).sort(dim=-1).values
        chosen[tokens, :, :idx.shape[-1]] = torch.where(idx < 1 << 30, idx, -1).to(I32)
    return {"chosen": chosen}


def _softmax_of(q, k, v, seen, d):
    """q [..., g, D], k and v [..., rows, D], seen [..., g or 1, rows]: outputs and logarithms of the sums."""
    x = (q @ k.transpose(-1, -2) * (1 / math.sqrt(d))).masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (x - m).exp()
    total = p.sum(-1, keepdim=True)
    return p @ v / total.clamp(min=1e-30), (total.log() + m)[..., 0]


def _run_attend(s):
    case = s["case"]
    br, hkv, d, g = case["block"], case["hkv"], case["d"], case["hq"] // case["hkv"]
    past = s["past"]
    other = torch.tensor([h for h in range(hkv) if h not in _past(case)], dtype=I64, device="cuda")
    b_of, i_of = _tokens(s)
    count = s["cu"][1:] - s["cu"][:-1]
    row = s["rows"][b_of].to(I64) - count[b_of][:, None] + i_of[:, None]  # [tokens, heads]
    q = s["q"].view(-1, hkv, g, d).to(F32)
    out = torch.zeros((s["total"], hkv, g, d), dtype=F32, device="cuda")
    lse = torch.zeros((s["total"], hkv, g), dtype=F32, device="cuda")
    rows_read = case["chosen"] * br
    some = max(1, (1 << 30) // (len(past) * rows_read * d * 4))
    for t in range(0, s["total"], some):
        part = slice(t, t + some)
        at = (s["chosen"][part].to(I64)[..., None] * br + torch.arange(br, device="cuda")).flatten(2)  # [tokens, past heads, rows]
        slot, ok = _slot(s, b_of[part][:, None, None], past[:, None], at)
        seen = ok & (at <= row[part][:, past, None])
        out[part, past], lse[part, past] = _softmax_of(q[part][:, past], _take(s, "k", slot), _take(s, "v", slot), seen[:, :, None], d)
    if len(other):
        p = torch.tensor(_policy(case), device="cuda")[other]
        start = row[:, other] // case["seg"] * case["seg"]
        first = (start - torch.where(p & 1 > 0, case["tail"], 0)).clamp(min=0)  # [tokens, other heads]
        if s["longest"] == 1:  # every token has a window of its own
            most = min(case["seg"] + case["tail"], s["max_rows"])
            some = max(1, (1 << 30) // (len(other) * most * d * 4))
            for t in range(0, s["total"], some):
                part = slice(t, t + some)
                at = first[part][..., None] + torch.arange(most, device="cuda")
                slot, ok = _slot(s, b_of[part][:, None, None], other[:, None], at)
                seen = ok & (at <= row[part][:, other, None])
                out[part, other], lse[part, other] = _softmax_of(q[part][:, other], _take(s, "k", slot), _take(s, "v", slot), seen[:, :, None], d)
        else:
            held, new = _sizes(case)
            for b in range(case["batch"]):  # the tokens of a sequence share the rows of all their windows
                if new[b] == 0:
                    continue
                t0 = sum(new[:b])
                lo = min(_window(case, int(x), held[b]) for x in case["policy"] if not int(x) & 2)
                at = torch.arange(lo, held[b] + new[b], device="cuda").expand(len(other), -1)
                slot, ok = _slot(s, torch.full_like(at, b), other[:, None], at)
                k, v = _take(s, "k", slot), _take(s, "v", slot)
                for t in range(t0, t0 + new[b], 256):
                    part = slice(t, min(t + 256, t0 + new[b]))
                    seen = ok[:, None] & (at[:, None] <= row[part, other].T[..., None]) & (at[:, None] >= first[part].T[..., None])
                    x = q[part][:, other].permute(1, 2, 0, 3).reshape(len(other), -1, d)  # [heads, g tokens, D]
                    y, z = _softmax_of(x, k, v, seen.repeat(1, g, 1), d)
                    out[part, other] = y.view(len(other), g, -1, d).permute(2, 0, 1, 3)
                    lse[part, other] = z.view(len(other), g, -1).permute(2, 0, 1)
    return {"out": out.to(s["out"].dtype).view(s["out"].shape), "lse": lse.view(s["lse"].shape)}


# --------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------
def _handles(s):
    """What a program keeps beside its cache: configuration, the description of pool and blocks, a workspace."""
    if "cfg" not in s:
        import paper_2605_11744_amd as sa
        case = s["case"]
        s["sa"] = sa
        s["cfg"] = sa.make_config(batch=case["batch"], n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["d"],
                                  seg_len=case["seg"], tail_len=case["tail"], kv_policy=_policy(case), out_fp32=case.get("f32", False))
        s["pages"] = sa.make_pages(k=s["k"], v=s["v"], table=s["table"], max_pages=s["most"], page_rows=case["page"],
                                   n_pages=s["k"].shape[0], per_head=case["per_head"], e4m3=case.get("e4m3", False),
                                   k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
        if "block" in case:
            s["blocks"] = sa.make_blocks(block_rows=case["block"], bounds=s["bounds"], scale=s["scale"])
        need = {"reserve": lambda: sa.seg_kv_paged_reserve_workspace_bytes(s["cfg"], s["pages"]),
                "choose": lambda: sa.seg_kv_paged_choose_workspace_bytes(s["cfg"], s["pages"], s["blocks"], s["total"], s["max_rows"],
                                                                         case["chosen"]),
                "attend": lambda: sa.seg_attn_paged_chosen_workspace_bytes(s["cfg"], s["pages"], s["blocks"], s["total"], s["longest"],
                                                                           s["max_rows"], case["chosen"])}.get(case["op"], lambda: 0)()
        s["workspace"], s["workspace_bytes"] = torch.empty(max(1, need), dtype=U8, device="cuda"), need
    return s["sa"], s["cfg"], torch.cuda.current_stream().cuda_stream


def _call(s):
    case = s["case"]
    sa, cfg, st = _handles(s)
    cu = s["cu"] if s["longest"] > 1 or s["total"] != case["batch"] else None  # None: one token of every sequence
    if case["op"] == "reserve":
        sa.seg_kv_paged_reserve(cfg, s["pages"], s["users"], cu, s["total"], s["longest"], s["held"], s["granted"], s["slots"],
                                s["workspace"], s["workspace_bytes"], newest_only=case["newest"], stream=st)
        return {"users": s["users"], "table": s["table"], "granted": s["granted"], "slots": s["slots"]}
    if case["op"] == "release":
        sa.seg_kv_paged_release(cfg, s["pages"], s["users"], s["rows"], stream=st)
        return {"users": s["users"], "table": s["table"]}
    if case["op"] == "summarize":
        sa.seg_kv_paged_summarize(cfg, s["pages"], s["blocks"], s["held"], s["rows"], s["longest"], stream=st)
        return {"bounds": s["bounds"], "scale": s["scale"]}
    if case["op"] == "choose":
        sa.seg_kv_paged_choose(cfg, s["pages"], s["blocks"], s["q"], cu, s["total"], s["longest"], s["rows"], s["max_rows"], case["chosen"],
                               case["first"], case["recent"], s["chosen"], s["workspace"], s["workspace_bytes"], stream=st)
        return {"chosen": s["chosen"]}
    sa.seg_attn_paged_chosen(cfg, s["pages"], s["blocks"], s["q"], cu, s["total"], s["longest"], s["rows"], s["max_rows"], s["chosen"],
                             case["chosen"], s["out"], s["lse"], s["workspace"], s["workspace_bytes"], stream=st)
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if "kept0" in state:  # the call works in place: tables and counts as they were, so that every pass has the same to do
        state["kept"].copy_(state["kept0"])
    if own:
        return _call(state)
    return {"reserve": _run_reserve, "release": _run_release, "summarize": _run_summarize, "choose": _run_choose,
            "attend": _run_attend}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# --------------------------------------------------------------------------------------------------
def work(case):
    B, hq, hkv, d, R = case["batch"], case["hq"], case["hkv"], case["d"], case["page"]
    held, new = _sizes(case)
    both, per_head = [a + b for a, b in zip(held, new)], hkv if case["per_head"] else 1
    past, most = _past(case), max(1, max(-(-n // R) for n in both))
    if case["op"] == "reserve":
        lo = [[max(a, _window(case, p, z - 1)) if case["newest"] else a for p in _policy(case)] for a, z in zip(held, both)]
        need = [sum(max(0, -(-z // R) - max(-(-a // R), x // R)) for x in (row if case["per_head"] else [min(row)]))
                for a, z, row in zip(held, both, lo)]
        taken = int(sum(need) * (0.6 if case["short"] else 1.0))
        named = sum(-(-a // R) - min(_window(case, p, a - 1) // R, -(-a // R)) for a in held for p in (_policy(case) if case["per_head"] else [2]))
        return {"bytes": 4 * (named + 3 * sum(need)) + 16 * taken + 8 * B * hkv + 8 * B + 8 * sum(new) * hkv, "flops": 0}
    if case["op"] == "release":
        return {"bytes": 4 * B * per_head * most + 4 * B * hkv, "flops": 0}
    row = 2 * (d + 1) if case.get("e4m3") else 4 * d  # bytes of a row's keys and values in the pages of one head
    br = case["block"]
    if case["op"] == "summarize":
        blocks = sum(z // br - a // br for a, z in zip(held, both)) * len(past)
        return {"bytes": blocks * (br * row // 2 + 2 * d + 1) + 8 * B * hkv, "flops": 2.0 * blocks * br * d}
    if case["op"] == "choose":
        scored = sum(m * max(0, a // br + 1 - case["first"] - case["recent"]) for a, m in zip(held, new) if a // br + 1 > case["chosen"])
        read = sum(max(0, z // br + 1 - case["first"] - case["recent"]) for z, m in zip(both, new) if m and z // br + 1 > case["chosen"])
        return {"bytes": len(past) * (read * (2 * d + 1) + sum(new) * (2 * d * hq // hkv + 4 * case["chosen"])),
                "flops": 4.0 * scored * len(past) * d * hq // hkv}
    seen, read = 0, 0  # (token, row) pairs, and rows that some token of the sequence reads
    for a, m in zip(held, new):
        if m == 0:
            continue
        mine = min(case["chosen"] * br, a + m)
        seen += m * mine * len(past)
        read += min(m * mine, a + m) * len(past)
        for p in _policy(case):
            if not p & 2:
                seen += sum(a + i + 1 - _window(case, p, a + i) for i in range(m))
                read += a + m - _window(case, p, a)
    return {"bytes": read * row + sum(new) * hq * ((6 if case["f32"] else 4) * d + 4) + 4 * sum(new) * len(past) * case["chosen"],
            "flops": 4.0 * seen * (hq // hkv) * d}


def exact(case, seed):
    if case["op"] != "attend":
        return None  # whole numbers: bounds and scores have no rounding that an order could change
    s = prepare(case, seed)
    hkv, d, br, g = case["hkv"], case["d"], case["block"], case["hq"] // case["hkv"]
    held, new = _sizes(case)
    out = torch.zeros((s["total"], hkv, g, d), dtype=F64, device="cuda")
    lse = torch.full((s["total"], hkv, g), -math.inf, dtype=F64, device="cuda")
    for b, (a, m) in enumerate(zip(held, new)):
        t0 = sum(new[:b])
        for h, p in enumerate(_policy(case)):
            lo = _window(case, p, a)
            at = torch.arange(lo, a + m, device="cuda")
            if m == 0:
                continue
            slot, _ = _slot(s, torch.full_like(at, b), torch.full_like(at, h), at)
            k, v = _take(s, "k", slot, F64), _take(s, "v", slot, F64)
            for t in range(0, m, 128):
                i = torch.arange(t, min(m, t + 128), device="cuda")
                if p & 2:  # a row counts where its block is listed
                    lists = s["chosen"][t0 + i, _past(case).index(h)].to(I64)
                    blocks = torch.zeros((len(i), (a + m) // br + 2), dtype=torch.bool, device="cuda")
                    blocks.scatter_(1, torch.where(lists < 0, blocks.shape[1] - 1, lists), True)
                    blocks[:, -1] = False
                    seen = blocks[:, at // br]
                else:
                    start = (a + i) // case["seg"] * case["seg"] - (case["tail"] if p & 1 else 0)
                    seen = at >= start[:, None]
                seen &= at <= (a + i)[:, None]
                for j in range(g):
                    x = (s["q"].view(-1, hkv, g, d)[t0 + i, h, j].to(F64) @ k.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
                    z = torch.logsumexp(x, -1)
                    lse[t0 + i, h, j] = z
                    out[t0 + i, h, j] = (x - z[:, None]).exp() @ v
    return {"out": out.view(-1, case["hq"], d), "lse": lse.view(-1, case["hq"])}
