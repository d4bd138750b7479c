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
