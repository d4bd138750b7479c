"""Performance cases of libsegattn's operators around a paged cache: what a serving or training program
calls when keys and values live in pages of a pool instead of one arena per layer.

    rotate   seg_rope_rotate: queries and keys turned by their positions (pairs in halves or interleaved,
             part of the head, frequencies scaled for long contexts), or gradients turned back
    append   seg_kv_paged_append: new tokens' queries and keys turned, keys and values written into the
             pages of their sequences, in bf16 or as e4m3 with a power-of-two scale per row
    decode   seg_attn_decode_paged: attention of one new token per sequence over the pages, and, where the
             cache keeps it, the weight that every row has received so far
    evict    seg_kv_paged_evict: of every head that holds more than `keep` rows the rows with the largest
             accumulated weight stay (the newest and the first ones always), and move into the freed places

`policy` has a digit per KV head: 0 own segment only, 1 carried tail, 2 past, 3 tail and past.  A head's
window is the one that the other attention calls of the library give the token.  Values are N(0, 1) rounded
to bf16, as in every workload of this repository.
"""
import math

import torch

own = False

BF16, F32, F64, I32, I64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def listed():
    return [
        # Queries and keys of a generation step of a small server: 16 tokens, the smallest call.
        {"name": "rotate_step", "op": "rotate", "batch": 16, "rows": 1, "hq": 32, "hkv": 8, "d": 128, "rotary": 128,
         "interleaved": False, "scaling": "none", "inverse": False, "f32": False, "fused": True},
        # A layer's 32K prompt in a context eight times the trained one.
        {"name": "rotate_32k", "op": "rotate", "batch": 1, "rows": 32768, "hq": 32, "hkv": 8, "d": 128, "rotary": 128,
         "interleaved": False, "scaling": "rotations", "inverse": False, "f32": False, "fused": False},
        # Training: fp32 gradients of dq and dk turned back, half of the head in neighbouring pairs.
        {"name": "rotate_grad", "op": "rotate", "batch": 3, "rows": 5003, "hq": 16, "hkv": 4, "d": 128, "rotary": 64,
         "interleaved": True, "scaling": "index", "inverse": True, "f32": True, "fused": False},
        # A generation step of 48 sequences: one token each, turned and written into pages of 64 rows.
        {"name": "append_step", "op": "append", "batch": 48, "lo": 1, "hi": 1, "held_lo": 500, "held_hi": 9000, "hq": 32,
         "hkv": 8, "d": 128, "page": 64, "per_head": False, "e4m3": False, "token_major": False, "rotary": 128,
         "interleaved": False},
        # Prompts of different lengths handed to an 8-bit cache after a prefill, small pages.
        {"name": "append_prompts_e4m3", "op": "append", "batch": 7, "lo": 61, "hi": 6001, "held_lo": 0, "held_hi": 900,
         "hq": 32, "hkv": 8, "d": 128, "page": 16, "per_head": False, "e4m3": True, "token_major": False, "rotary": 128,
         "interleaved": False},
        # Short conversations of a small multi-head layer, one sequence empty: latency counts.
        {"name": "decode_short", "op": "decode", "batch": 5, "lo": 0, "hi": 300, "hq": 8, "hkv": 8, "d": 64, "seg": 512,
         "tail": 128, "policy": "22222222", "page": 16, "per_head": False, "e4m3": False, "mass": False},
        # One user's generation behind 22.5K tokens: the window has to be split to fill the card.
        {"name": "decode_one", "op": "decode", "batch": 1, "lo": 22531, "hi": 22531, "hq": 32, "hkv": 8, "d": 128,
         "seg": 4096, "tail": 1024, "policy": "33331111", "page": 64, "per_head": False, "e4m3": False, "mass": False},
        # A server's step under segmented execution: contexts of 4K to 64K, a quarter of the KV heads long-range,
        # pages per head; the other heads' pages before their window are gone.
        {"name": "decode_segmented", "op": "decode", "batch": 64, "lo": 4097, "hi": 65536, "hq": 32, "hkv": 8, "d": 128,
         "seg": 4096, "tail": 1024, "policy": "33111111", "page": 64, "per_head": True, "e4m3": False, "mass": False},
        # Whole histories of 4K to 64K in bf16, every head long-range: the largest call.
        {"name": "decode_long", "op": "decode", "batch": 32, "lo": 4001, "hi": 65536, "hq": 32, "hkv": 8, "d": 128,
         "seg": 4096, "tail": 1024, "policy": "22222222", "page": 64, "per_head": False, "e4m3": False, "mass": False},
        # An 8-bit cache that is going to be evicted from: the step also adds up what every row receives.
        {"name": "decode_e4m3_mass", "op": "decode", "batch": 24, "lo": 1000, "hi": 32768, "hq": 32, "hkv": 8, "d": 128,
         "seg": 4096, "tail": 1024, "policy": "22222222", "page": 32, "per_head": False, "e4m3": True, "mass": True},
        # Back to a budget of 1024 rows after some hundred generated tokens.
        {"name": "evict_step", "op": "evict", "batch": 4, "lo": 1100, "hi": 1279, "keep": 1024, "recent": 256, "first": 4,
         "hq": 32, "hkv": 8, "d": 128, "page": 64, "per_head": False, "e4m3": False},
        # Long prompts cut to at most 16K rows of every head after their prefill, pages per head.
        {"name": "evict_prompts", "op": "evict", "batch": 12, "lo": 9000, "hi": 32768, "keep": 16384, "recent": 512,
         "first": 4, "hq": 32, "hkv": 8, "d": 128, "page": 64, "per_head": True, "e4m3": False},
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (16, 4, 128), (8, 8, 128), (16, 2, 128), (4, 4, 64), (16, 4, 64), (32, 8, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "decode", "decode", "decode", "evict"])
    hq, hkv, d = rng.choice(HEADS)
    c = {"op": op, "hq": hq, "hkv": hkv, "d": d}
    page, per_head, e4m3 = rng.choice([16, 24, 32, 64, 128, 256]), rng.random() < 0.3, rng.random() < 0.4
    if op == "rotate":
        rows = _log_int(rng, 1, 30000)
        c.update(batch=1 if rows > 9000 else rng.randint(1, 3) if rows > 50 else rng.randint(1, 64), rows=rows,
                 rotary=d // rng.choice([1, 1, 2, 4]), interleaved=rng.random() < 0.4,
                 scaling=rng.choice(["none", "linear", "rotations", "index"]), inverse=rng.random() < 0.4,
                 f32=rng.random() < 0.3, fused=rng.random() < 0.4)
    elif op == "append":
        step = rng.random() < 0.5
        hi = 1 if step else _log_int(rng, 8, 5000)
        held = _log_int(rng, 10, 6000)
        c.update(batch=_log_int(rng, 1, 100) if step else rng.randint(1, 8), lo=1 if step else rng.randint(0, hi // 2), hi=hi,
                 held_lo=held // rng.choice([1, 3, 10]), held_hi=held, page=page, per_head=per_head, e4m3=e4m3,
                 token_major=rng.random() < 0.3 and not per_head, rotary=d // rng.choice([1, 1, 2]),
                 interleaved=rng.random() < 0.3)
    elif op == "decode":
        hi = _log_int(rng, 5, 65000)
        mass = rng.random() < 0.3
        past = rng.choice([hkv, hkv, max(1, hkv // 4)])
        c.update(batch=rng.randint(1, max(1, min(64, 900000 // hi))), lo=hi // rng.choice([1, 2, 4, 50]), hi=hi,
                 seg=rng.choice([512, 1000, 4096]), tail=rng.choice([0, 128, 512]),
                 policy=rng.choice("23") * past + "1" * (hkv - past), page=page, per_head=per_head, e4m3=e4m3, mass=mass)
    else:
        keep = _log_int(rng, 60, 15000)
        more = _log_int(rng, 4, 2 * keep)
        c.update(batch=rng.randint(1, max(1, min(16, 150000 // (keep + more)))), lo=keep + more // 4, hi=keep + more, keep=keep,
                 recent=rng.randint(0, keep // 2), first=rng.choice([0, 4]), page=page, per_head=per_head, e4m3=e4m3)
    return c


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
THETA, FACTOR, TRAINED, LOW, HIGH = 500000.0, 8.0, 8192.0, 1.0, 4.0


def _lengths(n, lo, hi):
    """n lengths spread over lo..hi: both ends, then multiples of the golden ratio."""
    return [lo if i == 0 else hi if i == 1 else lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _policy(case):
    return [int(x) for x in case.get("policy", "2" * case["hkv"])]


def _first(case, n):
    """[B][Hkv] first visible row of every head for sequences that hold n[b] rows, the newest token's among them."""
    got = []
    for rows in n:
        start = max(0, rows - 1) // case["seg"] * case["seg"]
        got.append([0 if p & 2 else max(0, start - case["tail"]) if p & 1 else start for p in _policy(case)])
    return got


def _frequencies(case):
    """The frequency of every pair, in radians per position, and what the turned pairs are multiplied by."""
    n = case["rotary"]
    base, scaling, magnitude = [THETA ** (-2.0 * i / n) for i in range(n // 2)], case.get("scaling", "none"), 1.0
    if scaling == "linear":
        got = [f / FACTOR for f in base]
    elif scaling == "rotations":  # by how often a pair turns within the trained length
        kept = [min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW))) for f in base]
        got = [f * (k + (1 - k) / FACTOR) for f, k in zip(base, kept)]
    elif scaling == "index":  # by the pair's place between those that turn HIGH and LOW times
        at = [n * math.log(TRAINED / (2 * math.pi * r)) / (2 * math.log(THETA)) for r in (HIGH, LOW)]
        a, b = max(0, math.floor(at[0])), min(n - 1, math.ceil(at[1]))
        kept = [1 - min(1.0, max(0.0, (i - a) / max(b - a, 1e-3))) for i in range(n // 2)]
        got = [f * (k + (1 - k) / FACTOR) for f, k in zip(base, kept)]
        magnitude = 1.25
    else:
        got = base
    return got, magnitude


def _normal(g, shape, dtype=BF16):
    return torch.randn(shape, generator=g, device="cuda", dtype=F32 if dtype == F32 else BF16)


def _pages(case, s, g, first, rows, seed):
    """A pool whose pages lie in any order, and the table that names those of rows first..rows of every head."""
    B, H, R = case["batch"], case["hkv"], case["page"]
    heads = 1 if case["per_head"] else H
    most = max(1, max(-(-n // R) for n in rows))
    n = torch.tensor(rows, dtype=I64)[:, None].expand(B, H)
    lo = torch.tensor(first, dtype=I64)
    if not case["per_head"]:
        n, lo = n[:, :1], lo.min(dim=1, keepdim=True).values
    at = torch.arange(most)
    held = ((at >= (lo // R)[..., None]) & (at < (-(-n // R))[..., None])).cuda()
    used = int(held.sum())
    total = used + 3
    table = torch.full(held.shape, -1, dtype=I32, device="cuda")
    table[held] = torch.randperm(total, generator=g, device="cuda")[:used].to(I32)
    s["table"] = table if case["per_head"] else table[:, 0].contiguous()
    shape = (total, heads, R, case["d"])
    stored = (total, R, heads, case["d"]) if case.get("token_major") else shape

    def pool():
        x = _normal(g, stored)
        x = x.to(E4M3).view(U8) if case["e4m3"] else x
        return x.permute(0, 2, 1, 3) if case.get("token_major") else x

    s["k"], s["v"] = pool(), pool()
    if case["e4m3"]:
        s["k_scale"], s["v_scale"] = (torch.randint(125, 129, shape[:3], generator=g, device="cuda", dtype=U8) for _ in "kv")
    s["rows"] = torch.tensor(rows, dtype=I32)[:, None].expand(B, H).contiguous().cuda()
    return shape


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, B, hq, hkv, d = case["op"], case["batch"], case["hq"], case["hkv"], case["d"]
    s = {"case": case}
    if "rotary" in case:
        f, s["magnitude"] = _frequencies(case)
        s["frequencies"] = torch.tensor(f, dtype=F64, device="cuda")
    if op == "rotate":
        n, t = B * case["rows"], F32 if case["f32"] else BF16
        if case["fused"]:  # as a projection leaves them: queries, keys and values of a token side by side
            x = _normal(g, (n, hq + 2 * hkv, d), t)
            s["q"], s["k"] = x[:, :hq], x[:, hq:hq + hkv]
        else:
            s["q"], s["k"] = _normal(g, (n, hq, d), t), _normal(g, (n, hkv, d), t)
        s["pos0"] = torch.randint(0, 50000, (B,), generator=g, device="cuda", dtype=I64)
        s["q_out"], s["k_out"] = (torch.empty((n, h, d), dtype=t, device="cuda") for h in (hq, hkv))
        return s
    if op == "append":
        new, held = _lengths(B, case["lo"], case["hi"]), _lengths(B, case["held_lo"], case["held_hi"])
        both = [a + b for a, b in zip(new, held)]
        shape = _pages(case, s, g, [[0] * hkv] * B, both, seed)
        s["rows"] -= torch.tensor(new, dtype=I32, device="cuda")[:, None]
        n = sum(new)
        s["cu"] = torch.tensor([sum(new[:i]) for i in range(B + 1)], dtype=I32, device="cuda")
        s["total"], s["longest"] = n, max(new)
        s["pos0"] = s["rows"][:, 0].to(I64) + torch.randint(0, 9000, (B,), generator=g, device="cuda")
        s["q"], s["nk"], s["nv"] = _normal(g, (n, hq, d)), _normal(g, (n, hkv, d)), _normal(g, (n, hkv, d))
        s["q_out"], s["rows_out"] = torch.empty_like(s["q"]), torch.empty_like(s["rows"])
        s["pos"] = torch.full(shape[:3], -1, dtype=I32, device="cuda")
        s["mass"] = torch.rand(shape[:3], generator=g, device="cuda")
        return s
    rows = _lengths(B, case["lo"], case["hi"])
    if op == "decode":
        shape = _pages(case, s, g, _first(case, rows), rows, seed)
        s["longest"] = max(1, max(rows))
        s["q"] = _normal(g, (B, hq, d))
        s["past"] = torch.tensor([bool(p & 2) for p in _policy(case)], device="cuda")
        s["carried"] = torch.tensor([case["tail"] if p & 1 else 0 for p in _policy(case)], device="cuda")
        s["out"] = torch.empty((B, hq, d), dtype=BF16, device="cuda")
        s["lse"] = torch.empty((B, hq), dtype=F32, device="cuda")
        if case["mass"]:
            s["mass"] = torch.rand(shape[:3], generator=g, device="cuda")
        return s
    shape = _pages(case, s, g, [[0] * hkv] * B, rows, seed)
    s["longest"] = max(rows)
    s["rows_out"] = torch.empty_like(s["rows"])
    # What a cache that was evicted from before holds: positions in any order below the budget, ascending above
    # it; weights that few rows have much of, and some rows none.
    n, R = shape[0] * shape[1] * shape[2], case["page"]
    kept = torch.zeros((2, n), dtype=I32, device="cuda")
    at = torch.arange(s["table"].shape[-1] * R, device="cuda")
    at = torch.rand((B, hkv, min(case["keep"], at.numel())), generator=g, device="cuda").argsort(-1), at
    at = torch.cat([at[0], at[1][case["keep"]:].expand(B, hkv, -1)], -1)
    slot, held = _slots(case, s, at.shape[-1])
    held &= torch.arange(at.shape[-1], device="cuda") < s["rows"][..., None]
    kept[0, slot[held]] = at[held].to(I32)
    kept[1] = (torch.rand(n, generator=g, device="cuda") - 0.05).clamp(min=0).pow(4).view(I32)
    s["kept0"], s["kept"] = kept, kept.clone()
    s["pos"], s["mass"] = s["kept"][0].view(shape[:3]), s["kept"][1].view(F32).view(shape[:3])
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------------
def _slots(case, s, n):
    """For rows 0..n-1 of every (sequence, head): the row's place among all rows of the pool's heads, and whether it has one."""
    R, H = case["page"], case["hkv"]
    at = torch.arange(n, device="cuda")
    page = s["table"][..., (at // R).clamp(max=s["table"].shape[-1] - 1)].to(I64)
    if case["per_head"]:
        slot = page * R + at % R
    else:
        page = page[:, None, :].expand(-1, H, -1)
        slot = (page * H + torch.arange(H, device="cuda")[:, None]) * R + at % R
    return slot.clamp(min=0), (page >= 0) & (at < s["table"].shape[-1] * R)


def _take(case, pool, scale, slot, dtype):
    """The rows `slot` names, as numbers of `dtype`."""
    x = pool.reshape(-1, case["d"])[slot]
    return torch.ldexp(x.view(E4M3).to(dtype), (scale.reshape(-1)[slot].to(I32) - 127)[..., None]) if case["e4m3"] else x.to(dtype)


def _turn(s, x, position, inverse=False):
    """x [tokens, heads, D] with the pairs of its first `rotary` channels turned by position * frequency."""
    case, n = s["case"], s["case"]["rotary"]
    angle = position.to(F64)[:, None] * s["frequencies"]
    angle = -angle if inverse else angle
    c, sn = (s["magnitude"] * angle.cos()).to(F32)[:, None], (s["magnitude"] * angle.sin()).to(F32)[:, None]
    x = x.to(F32)
    y, rest = x[..., :n], x[..., n:]
    if case["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)
    else:
        a, b = y[..., :n // 2], y[..., n // 2:]
        y = torch.cat([a * c - b * sn, a * sn + b * c], -1)
    return torch.cat([y, rest], -1)


def _stored(x):
    """Rows in e4m3, and the power of two each has to be multiplied by: the smallest that leaves the row's largest value at most 448."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m == 0, torch.zeros_like(e), e - 9 + (m > 0.875).to(e.dtype))
    return torch.ldexp(x, -e[..., None]).to(F32).to(E4M3), (e + 127).to(U8)


def _run_rotate(s):
    case = s["case"]
    t = torch.arange(case["batch"] * case["rows"], device="cuda")
    position = s["pos0"][t // case["rows"]] + t % case["rows"]
    return {x: _turn(s, s[x], position, case["inverse"]).to(s[x].dtype) for x in "qk"}


def _new_tokens(s):
    """Sequence and position of every new token, and the place of its row among all rows of the pool's heads."""
    case = s["case"]
    R, H = case["page"], case["hkv"]
    t = torch.arange(s["total"], device="cuda")
    b = torch.searchsorted(s["cu"].to(I64), t, right=True) - 1
    i = t - s["cu"][b]
    row = s["rows"][b].to(I64) + i[:, None]
    head = torch.arange(H, device="cuda").expand(len(t), H)
    if case["per_head"]:
        return b, s["pos0"][b] + i, (s["table"][b[:, None], head, row // R].to(I64), torch.zeros_like(head), row % R)
    return b, s["pos0"][b] + i, (s["table"][b[:, None], row // R].to(I64), head, row % R)


def _held(s):
    """What the pool holds, 8-bit rows as the values that their bits stand for."""
    got = {x: s[x] for x in ("k", "v", "pos", "mass")}
    if s["case"]["e4m3"]:
        got |= {x: s[x].view(E4M3) for x in "kv"} | {x: s[x].view(E8M0) for x in ("k_scale", "v_scale")}
    return got


def _run_append(s):
    case = s["case"]
    b, position, at = _new_tokens(s)
    k, v = _turn(s, s["nk"], position), s["nv"]
    if case["e4m3"]:
        k, s["k_scale"][at] = _stored(k)
        v, s["v_scale"][at] = _stored(v.to(F32))
        k, v = k.view(U8), v.view(U8)
    s["k"][at], s["v"][at] = k.to(s["k"].dtype), v
    s["pos"][at] = position.to(I32)[:, None].expand(-1, case["hkv"])
    s["mass"][at] = 0.0
    rows = s["rows"] + (s["cu"][1:] - s["cu"][:-1])[:, None]
    return _held(s) | {"q": _turn(s, s["q"], position).to(BF16), "rows": rows}


def _run_decode(s):
    case = s["case"]
    B, hq, hkv, d, n = case["batch"], case["hq"], case["hkv"], case["d"], s["longest"]
    slot, held = _slots(case, s, n)
    at, rows = torch.arange(n, device="cuda"), s["rows"].to(I64)
    start = (rows - 1).clamp(min=0) // case["seg"] * case["seg"]
    first = torch.where(s["past"], 0, (start - s["carried"]).clamp(min=0))
    seen = held & (at >= first[..., None]) & (at < rows[..., None])
    q = s["q"].view(B, hkv, hq // hkv, d).to(F32)
    x = q @ _take(case, s["k"], s.get("k_scale"), slot, F32).transpose(-1, -2) * (1 / math.sqrt(d))
    x = x.masked_fill(~seen[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (x - m).exp()
    total = p.sum(-1, keepdim=True)
    out = p @ _take(case, s["v"], s.get("v_scale"), slot, F32) / total.clamp(min=1e-30)
    got = {"out": out.to(BF16).view(B, hq, d), "lse": (total.log() + m).view(B, hq)}
    if case["mass"]:
        w = (p / total.clamp(min=1e-30)).sum(2)
        w = w.masked_fill(~(seen & s["past"][:, None]), 0.0)
        s["mass"].view(-1).index_add_(0, slot.flatten(), w.flatten())
        got["mass"] = s["mass"]
    return got


def _run_evict(s):
    case = s["case"]
    n, keep = s["longest"], case["keep"]
    slot, held = _slots(case, s, n)
    at, rows = torch.arange(n, device="cuda"), s["rows"].to(I64)
    held = held & (at < rows[..., None])
    pos, mass = s["pos"].view(-1)[slot].to(I64), s["mass"].view(-1)[slot]
    newest = pos.masked_fill(~held, -1).amax(-1, keepdim=True)
    rank = mass.masked_fill((pos > newest - case["recent"]) | (pos < case["first"]), math.inf).masked_fill(~held, -1.0)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = torch.zeros_like(held).scatter_(-1, order, True) & held
    over = (rows > keep)[..., None]
    to = slot[~kept & (at < keep) & over]  # both in the order of sequence, head and row: as many of the one as of the other
    of = slot[kept & (at >= keep) & over]
    for name in ("k", "v", "k_scale", "v_scale", "pos", "mass"):
        if name in s:
            x = s[name].view(-1, case["d"]) if name in "kv" else s[name].view(-1)
            x[to] = x[of]
    return _held(s) | {"rows": rows.clamp(max=keep).to(I32)}


# --------------------------------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------------------------------
def _handles(s):
    """What a program keeps beside its cache: configuration, rotation, the description of the pool, a workspace."""
    if "cfg" not in s:
        import paper_2605_11744_amd as sa
        case = s["case"]
        s["sa"] = sa
        s["cfg"] = sa.make_config(batch=case["batch"], n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["d"],
                                  seg_len=case.get("seg", 4096), tail_len=case.get("tail", 0), kv_policy=_policy(case))
        if "rotary" in case:
            scaling = {"none": sa.SEGATTN_ROPE_PLAIN, "linear": sa.SEGATTN_ROPE_LINEAR, "rotations": sa.SEGATTN_ROPE_BY_ROTATIONS,
                       "index": sa.SEGATTN_ROPE_BY_INDEX}[case.get("scaling", "none")]
            s["rope"] = sa.make_rope(theta=THETA, rotary_dim=case["rotary"], interleaved=case["interleaved"], scaling=scaling,
                                     factor=FACTOR, trained_len=TRAINED, low=LOW, high=HIGH, magnitude=_frequencies(case)[1])
        if "table" in s:
            k = s["k"]
            s["pages"] = sa.make_pages(k=k, v=s["v"], table=s["table"], max_pages=s["table"].shape[-1], page_rows=case["page"],
                                       n_pages=k.shape[0], per_head=case["per_head"], e4m3=case["e4m3"],
                                       page_stride=k.stride(0), head_stride=k.stride(1), row_stride=k.stride(2),
                                       k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), mass=s.get("mass"), pos=s.get("pos"))
            need = {"decode": lambda: sa.seg_attn_decode_paged_workspace_bytes(s["cfg"], s["pages"], s["longest"], case.get("mass", False)),
                    "evict": lambda: sa.seg_kv_paged_evict_workspace_bytes(s["cfg"], s["pages"], s["longest"], case["keep"]),
                    "append": lambda: 0}[case["op"]]()
            s["workspace"], s["workspace_bytes"] = torch.empty(max(1, need), dtype=U8, device="cuda"), need
    return s["sa"], s["cfg"], torch.cuda.current_stream().cuda_stream


def _call(s):
    case = s["case"]
    sa, cfg, st = _handles(s)
    if case["op"] == "rotate":
        sa.seg_rope_rotate(cfg, s["rope"], s["q"], s["k"], case["rows"], s["q_out"], s["k_out"], pos0=s["pos0"],
                           inverse=case["inverse"], fp32=case["f32"], q_stride=s["q"].stride(0), k_stride=s["k"].stride(0), stream=st)
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["op"] == "append":
        sa.seg_kv_paged_append(cfg, s["pages"], s["rope"], s["q"], s["nk"], s["nv"], s["cu"], s["total"], s["longest"], s["pos0"],
                               s["rows"], s["q_out"], s["rows_out"], stream=st)
        return _held(s) | {"q": s["q_out"], "rows": s["rows_out"]}
    if case["op"] == "decode":
        sa.seg_attn_decode_paged(cfg, s["pages"], s["q"], s["rows"], s["longest"], s["out"], s["lse"], s["workspace"],
                                 s["workspace_bytes"], accumulate=case["mass"], stream=st)
        return {"out": s["out"], "lse": s["lse"]} | ({"mass": s["mass"]} if case["mass"] else {})
    sa.seg_kv_paged_evict(cfg, s["pages"], s["rows"], s["longest"], case["keep"], case["recent"], case["first"], s["rows_out"],
                          s["workspace"], s["workspace_bytes"], stream=st)
    return _held(s) | {"rows": s["rows_out"]}


def run(state):
    if state["case"]["op"] == "evict":  # the call works in place: positions and weights as they were, so that every pass has the same to do
        state["kept"].copy_(state["kept0"])
    if own:
        return _call(state)
    return {"rotate": _run_rotate, "append": _run_append, "decode": _run_decode, "evict": _run_evict}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# --------------------------------------------------------------------------------------------------
def work(case):
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if case["op"] == "rotate":
        values = B * case["rows"] * (hq + hkv) * d
        return {"bytes": 2 * values * (4 if case["f32"] else 2) + 8 * B, "flops": 3 * values * case["rotary"] / d}
    row = 2 * (d + 1) if case["e4m3"] else 4 * d  # bytes of a row's keys and values in the pages of one head
    if case["op"] == "append":
        n = sum(_lengths(B, case["lo"], case["hi"]))
        return {"bytes": n * (4 * hq * d + hkv * (4 * d + row + 8)) + 8 * B * hkv + 12 * B,
                "flops": 3 * n * (hq + hkv) * case["rotary"]}
    rows = _lengths(B, case["lo"], case["hi"])
    if case["op"] == "decode":
        seen = sum(n - f for n, first in zip(rows, _first(case, rows)) for f in first)
        kept = sum(rows) * sum(p >> 1 for p in _policy(case)) if case["mass"] else 0
        return {"bytes": seen * row + 8 * kept + B * hq * (4 * d + 4), "flops": 4.0 * seen * (hq // hkv) * d}
    keep, sure = case["keep"], case["recent"]
    # rows that stay and lie behind the budget: the newest ones, and of the others their share
    moved = sum(min(n - keep, sure) + (keep - sure) * max(0, n - keep - sure) / (n - sure) for n in rows if n > keep)
    return {"bytes": hkv * (8 * sum(n for n in rows if n > keep) + moved * (2 * row + 16) + 8 * B), "flops": 0}


def _exact_turned(case, x, position, inverse=False):
    """As the definition has it: a pair is a complex number, its turning a product with magnitude * exp(i angle)."""
    n = case["rotary"]
    f, magnitude = _frequencies(case)
    x = x.to(F64).clone()
    i = torch.arange(n // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + n // 2)
    angle = torch.outer(position.to(F64), torch.tensor(f, dtype=F64, device=x.device)) * (-1.0 if inverse else 1.0)
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    x[..., a], x[..., b] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if case["op"] == "rotate":
        position = torch.cat([p + torch.arange(case["rows"], device="cuda") for p in s["pos0"]])
        return {x: _exact_turned(case, s[x], position, case["inverse"]) for x in "qk"}
    if case["op"] == "append":
        got = {x: None for x in ("q", "k", "v", "k_scale", "v_scale", "pos", "rows", "mass")}
        b, position, at = _new_tokens(s)
        got["q"], new = _exact_turned(case, s["q"], position), {"k": _exact_turned(case, s["nk"], position), "v": s["nv"].to(F64)}
        for name, x in new.items():
            if case["e4m3"]:  # e4m3 has four significant bits down to 2^-6, and steps of 2^-9 below
                pool, scales = s[name].view(E4M3).to(F64), torch.exp2(s[name + "_scale"].to(F64) - 127)
                most = x.abs().amax(-1)
                scale = torch.exp2(torch.ceil(torch.log2(torch.where(most > 0, most, 448.0) / 448.0)))
                y = x / scale[..., None]
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                pool[at], scales[at] = (y / step).round() * step, scale
                got[name], got[name + "_scale"] = pool, scales
            else:
                got[name] = s[name].to(F64)
                got[name][at] = x
        return got
    if case["op"] == "evict":
        return None  # nothing is computed: rows move as they are
    out, lse = torch.zeros((B, hq, d), dtype=F64, device="cuda"), torch.full((B, hq), -math.inf, dtype=F64, device="cuda")
    mass = s["mass"].to(F64) if case["mass"] else None
    rows, slot = _lengths(B, case["lo"], case["hi"]), _slots(case, s, s["longest"])[0]
    for b, first in enumerate(_first(case, rows)):
        for h in range(hkv):
            at = slot[b, h, first[h]:rows[b]]
            if at.numel() == 0:
                continue
            k, v = (_take(case, s[x], s.get(x + "_scale"), at, F64) for x in "kv")
            x = s["q"].view(B, hkv, -1, d)[b, h].to(F64) @ k.T / math.sqrt(d)
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            lse[b, heads] = torch.logsumexp(x, -1)
            p = (x - lse[b, heads, None]).exp()
            out[b, heads] = p @ v
            if case["mass"] and _policy(case)[h] & 2:
                mass.view(-1)[at] += p.sum(0)
    return {"out": out, "lse": lse} | ({"mass": mass} if case["mass"] else {})
