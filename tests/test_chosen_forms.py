"""The form that attention over chosen blocks and the reservation of pages take, asked from the library's rules on the CPU (tests/host/chosen_forms.hip): that the GPU tests
written for a form have shapes that take it."""
import os
import shutil
import subprocess

import pytest

import paper_2605_11744_amd as sa
from conftest import ROOT


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    sa.lib()  # built, and says so if not
    pkg = os.path.join(ROOT, "paper_2605_11744_amd")
    exe = tmp_path_factory.mktemp("forms") / "chosen_forms"
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(pkg, "csrc"), os.path.join(ROOT, "tests", "host", "chosen_forms.hip"),
                    "-L", pkg, "-lsegattn", "-Wl,-rpath," + pkg, "-o", str(exe)], check=True, capture_output=True, timeout=600)

    def ask(lines):
        out = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=600)
        assert out.returncode == 0, out.stdout + out.stderr
        got = [x.split() for x in out.stdout.splitlines()]
        assert len(got) == len(lines)
        return [x[0] if len(x) == 1 else dict(listed=x[0], part=int(x[1]), windows=x[2], workgroups=int(x[3]), laid_out=int(x[4]), asked=int(x[5])) for x in got]

    return ask


def line(*, d, g, policy, seg, tail, new, most, block, chosen, e4m3=False, out_fp32=True, total=None):
    return (f"{d} {g * len(policy)} {len(policy)} {''.join(map(str, policy))} {seg} {tail} {len(new)} {total or sum(new)} {max(new)} {most} {block} {chosen} "
            f"{int(e4m3)} {int(out_fp32)}")


def test_chunks_whose_columns_are_compared_share_blocks_and_tiles(forms):
    from test_gpu_sparse_columns import BLOCK, CHUNKS, HELD, POLICY, SEG, TAIL
    got = forms([line(d=d, g=g, policy=POLICY, seg=SEG, tail=TAIL, new=[n], most=-(-(HELD + n) // BLOCK) * BLOCK, block=BLOCK, chosen=chosen, e4m3=e4m3, out_fp32=f)
                 for d, g, e4m3, n, chosen in CHUNKS for f in (True, False)])
    assert [(x["listed"], x["windows"]) for x in got] == [("blocks", "shares")] * len(got)


def test_a_thread_does_not_go_through_many_entries(forms):
    """Few sequences with many entries each: one workgroup, a thread a sequence, takes up to a millisecond where four launches take 20 us."""
    ask = lambda heads, sequences, page_rows, per_head, new: forms([f"reserve {heads} {sequences} {page_rows} 9000 {per_head} {sequences * new} {new}"])[0]
    for many in ((1, 1, 1, 0, 2560), (8, 1, 16, 0, 320), (8, 1, 16, 1, 320), (8, 1, 1, 1, 320), (2, 1, 16, 0, 1280), (8, 8, 16, 1, 40)):
        assert ask(*many) == "four", many
    for step in ((8, 48, 64, 0, 1), (8, 256, 16, 1, 1), (8, 64, 64, 0, 5), (8, 8, 16, 0, 40), (2, 100, 16, 1, 1)):
        assert ask(*step) == "one", step


def _random_call(rng):
    """A call and the sizes of a smaller one with the same heads, types and blocks."""
    H = rng.choice([1, 2, 4, 8, 8, 16, 64])
    fixed = dict(d=rng.choice([64, 128]), g=rng.choice([1, 2, 4, 4, 7, 8, 16, 17, 40, 128]), policy=[rng.choice([0, 1, 2, 3]) for _ in range(H)],
                 seg=rng.choice([16, 64, 512, 4096]), tail=rng.choice([0, 5, 16]), block=rng.choice([16, 48, 64, 128, 512]), e4m3=rng.random() < 0.5,
                 out_fp32=rng.random() < 0.5)
    log = lambda lo, hi: min(hi, max(lo, int(lo * (hi / lo) ** rng.random() + 0.5)))
    B, longest = log(1, 300), rng.choice([1, log(1, 8), log(1, 60000)])
    big = dict(B=B, longest=longest, total=rng.randint(longest, min(B * longest, 400000)) if B * longest > longest else longest, most=log(1, 2000000),
               chosen=rng.choice([log(1, 64), log(1, 4096), log(1, 65536)]))
    big["total"] = max(big["total"], longest)
    small = dict(B=log(1, B), longest=log(1, longest), most=log(1, big["most"]), chosen=log(1, big["chosen"]))
    small = {x: (y if rng.random() < 0.6 else big[x]) for x, y in small.items()}
    hi = min(small["B"] * small["longest"], big["total"])
    small["total"] = log(small["longest"], hi)
    return fixed, big, small


def _call_line(fixed, size):
    new = [size["longest"]] + [0] * (size["B"] - 1)
    return line(**fixed, new=new, total=size["total"], most=size["most"], chosen=size["chosen"])


def test_a_workspace_covers_every_smaller_call(forms):
    """Which forms calls take changes with their sizes; a program allocates once, for its largest.  No form lays out more than is asked for."""
    import random
    rng = random.Random(11)
    calls = [_random_call(rng) for _ in range(4000)]
    large, little = (forms([_call_line(c[0], c[i]) for c in calls]) for i in (1, 2))
    for call, x, y in zip(calls, large, little):
        assert x["laid_out"] <= x["asked"] and y["laid_out"] <= y["asked"] <= x["asked"] <= 2.25 * 2 ** 30, (call, x, y)
    kinds = {(x["listed"], x["windows"]) for x in large + little}
    assert kinds == {(x, y) for x in ("blocks", "tokens") for y in ("shares", "units", "tokens")}
    # one batch, all of its lengths
    for policy in ([1] * 8, [2] * 8, [3, 3, 3, 3, 1, 1, 1, 1]):
        asked = [forms([line(d=128, g=4, policy=policy, seg=4096, tail=1024, new=[n] + [0] * (B - 1), most=131072, block=64, chosen=32)])[0]["asked"]
                 for B, n in ((1, 1), (1, 2), (1, 64), (2, 64), (2, 512), (2, 4096), (8, 4096), (8, 8192), (8, 16384), (8, 32768))]
        assert asked == sorted(asked), (policy, asked)


def test_the_room_for_a_choice_covers_every_smaller_one():
    sizes = [(n, rows, chosen) for n in (1, 17, 1000, 8192, 100000) for rows in (100, 90000, 100000, 131072, 4000000) for chosen in (4, 64)]
    cfg = sa.make_config(batch=100000, n_q_heads=32, n_kv_heads=8, head_dim=128, seg_len=4096, tail_len=1024, kv_policy=[2] * 8)
    pages = sa.make_pages(k=4096, v=4096, table=4096, max_pages=4000000 // 64, page_rows=64, n_pages=1)
    blocks = sa.make_blocks(block_rows=64, bounds=4096, scale=4096)
    need = {s: sa.seg_kv_paged_choose_workspace_bytes(cfg, pages, blocks, *s) for s in sizes}
    for s in sizes:
        assert need[s] > 0 and all(need[t] <= need[s] for t in sizes if all(x <= y for x, y in zip(t, s))), s


def test_windows_written_for_a_form_take_it(forms):
    from test_gpu_sparse import SHARED
    from test_gpu_sparse_forms import SHORT
    most = lambda new, held, block: -(-max(h + n for h, n in zip(held, new)) // block) * block
    lines, want = [], []
    for d, g, policy, seg, tail, (new, held), kind in SHORT:
        for e4m3 in (False, True):
            lines.append(line(d=d, g=g, policy=policy, seg=seg, tail=tail, new=new, total=sum(new) + (len(new) > 1), most=most(new, held, 16), block=16, chosen=4, e4m3=e4m3,
                              out_fp32=not e4m3))
            want.append(kind)
    for kind, d, g, out_fp32 in SHARED:
        new, held, block = [900, 1100, 0, 1], [1990, 3500, 100, 0], kind["block"]
        lines.append(line(d=d, g=g, policy=[1, 2, 0], seg=1000, tail=300, new=new, total=sum(new) + 2, most=most(new, [h + 1 for h in held], kind["page_rows"]), block=block,
                          chosen=4, e4m3=kind.get("e4m3", False), out_fp32=out_fp32))
        want.append("shares")
    for e4m3 in (False, True):
        lines.append(line(d=128, g=4, policy=[1, 2, 0], seg=1000, tail=300, new=[2000], most=3520, block=32, chosen=3, e4m3=e4m3))
        lines.append(line(d=128, g=16, policy=[1, 0, 1, 1, 0, 0, 1, 1], seg=200, tail=56, new=[2044, 6], most=2240, block=64, chosen=1, e4m3=e4m3, out_fp32=not e4m3))
        want += ["shares", "units"]
    got = forms(lines)
    assert [x["windows"] for x in got] == want


def test_long_chunks_written_for_listed_blocks_take_them_once(forms):
    from test_gpu_sparse import LONG
    lines = []
    for kind in LONG:
        e4m3 = kind.get("e4m3", False)
        new = [2600 if e4m3 else 1290, 0, 17]
        held, page = [700, 30, 2000], kind["page_rows"]
        lines += [line(d=128, g=2 if e4m3 else 4, policy=[2, 3], seg=64, tail=16, new=new, total=sum(new) + 3, chosen=16 if e4m3 else 8, e4m3=e4m3, out_fp32=f,
                       most=-(-(max(h + n for h, n in zip(held, new)) + 1) // page) * page, block=kind["block"]) for f in (False, True)]
    for d, g in ((64, 1), (64, 8), (128, 3), (128, 1)):
        new = [2600 if g == 8 else 1290, 0, 17]
        lines.append(line(d=d, g=g, policy=[2, 3], seg=64, tail=16, new=new, total=sum(new) + 3, chosen=16 if g == 8 else 8, most=-(-(700 + new[0] + 1) // 64) * 64, block=64))
    assert [x["listed"] for x in forms(lines)] == ["blocks"] * len(lines)


def test_reservations_written_for_a_form_take_it(forms):
    from test_gpu_sparse_forms import RESERVATIONS
    got = forms([f"reserve 3 {n} 16 9000 {per_head} {n * most // 2} {most}" for n, most in RESERVATIONS for per_head in (0, 1)])
    assert got == ["one", "one"] + ["four"] * 6
