"""seg_rope_rotate against its definition in 64 bits.

Error of a turned element: the angle is reduced in double and rounded to a float of at most half a turn (2^-26 turns =
9.4e-8 rad), sine and cosine are good to a few units of 2^-24, and the products and their sum add three
roundings: below 2^-20 of magnitude * (|a| + |b|), and half a step of the type it is stored in."""
import numpy as np
import pytest
import torch

import paper_2605_11744_amd as sa
import paged_ref as ref

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}

ROPES = [
    dict(theta=500000.0),
    dict(theta=10000.0, rotary_dim=32),
    dict(theta=10000.0, interleaved=True),
    dict(theta=1000.0, rotary_dim=48, interleaved=True, scaling=sa.SEGATTN_ROPE_LINEAR, factor=4.0),
    dict(theta=500000.0, scaling=sa.SEGATTN_ROPE_BY_ROTATIONS, factor=8.0, trained_len=8192.0, low=1.0, high=4.0, magnitude=1.25),
    dict(theta=10000.0, rotary_dim=64, scaling=sa.SEGATTN_ROPE_BY_INDEX, factor=16.0, trained_len=4096.0, low=1.0, high=32.0, magnitude=0.75),
    dict(theta=1.0, rotary_dim=16, inv_freq=[0.0, 1.0, -0.5, 3.25, 1e-9, 0.1, 0.01, 2.0]),
]


def _cfg(batch, hq, hkv, d):
    return sa.make_config(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seg_len=512, tail_len=64, kv_policy=[1] * hkv)


def _check(got, x, positions, rope, inverse=False, what=""):
    want, size = ref.turned(x.to(torch.float64).cpu(), positions, rope, inverse)
    err = (got.to(torch.float64).cpu() - want).abs()
    bound = want.abs() * HALF_STEP[x.dtype] * (1 + 2.0 ** -7) + size * 2.0 ** -20 + 1e-38
    n = rope.get("rotary_dim", 0) or x.shape[-1]
    assert (err <= bound).all(), f"{what}: {float((err - bound).max()):.3e} above the bound"
    assert torch.equal(ref.bits(got[..., n:]), ref.bits(x[..., n:])), f"{what}: channels behind the turned ones"


@pytest.mark.parametrize("rope", ROPES, ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items() if k != "inv_freq")[:60])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("batch,rows,hq,hkv,d", [(1, 1, 4, 4, 64), (3, 17, 6, 2, 128), (2, 1031, 8, 1, 64)])
def test_rotation_matches_the_definition(rope, dtype, batch, rows, hq, hkv, d):
    g = torch.Generator().manual_seed(rows)
    q, k = (torch.randn((batch * rows, h, d), generator=g).to(dtype).cuda() for h in (hq, hkv))
    pos0 = torch.randint(0, 1 << 20, (batch,), generator=g, dtype=torch.int64)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    sa.seg_rope_rotate(_cfg(batch, hq, hkv, d), sa.make_rope(**rope), q, k, rows, qo, ko, pos0=pos0.cuda(), fp32=dtype == torch.float32,
                       stream=torch.cuda.current_stream().cuda_stream)
    at = (pos0[:, None] + torch.arange(rows)).flatten()
    _check(qo, q, at, rope, what="q")
    _check(ko, k, at, rope, what="k")


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_projection_positions_per_row_and_in_place(inverse, interleaved):
    """q and k as slices of one [tokens, (Hq + 2 Hkv) D] tensor, positions in any order, a result in place."""
    n, hq, hkv, d = 203, 4, 2, 128
    rope = dict(theta=10000.0, rotary_dim=96, interleaved=interleaved)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((n, hq + 2 * hkv, d), generator=g).to(torch.bfloat16).cuda()
    pos = torch.randint(-50, 1 << 30, (n,), generator=g, dtype=torch.int64)
    before = x.clone()
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    wide = torch.full((n, hkv + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    sa.seg_rope_rotate(_cfg(1, hq, hkv, d), sa.make_rope(**rope), q, k, n, q, wide, pos=pos.cuda(), inverse=inverse, q_stride=x.stride(0),
                       k_stride=x.stride(0), q_out_stride=x.stride(0), k_out_stride=wide.stride(0), stream=torch.cuda.current_stream().cuda_stream)
    _check(x[:, :hq].contiguous(), before[:, :hq].contiguous(), pos, rope, inverse, "q in place")
    _check(wide[:, :hkv].contiguous(), before[:, hq:hq + hkv].contiguous(), pos, rope, inverse, "k")
    assert torch.equal(ref.bits(x[:, hq:]), ref.bits(before[:, hq:])) and (wide[:, hkv:] == 7.0).all()


def test_outputs_between_the_inputs_rows():
    """All four tensors are parts of one [tokens, 2 (Hq + Hkv) D] tensor; then outputs that begin where the inputs end."""
    n, hq, hkv, d, rope = 67, 4, 2, 64, dict(theta=10000.0)
    x = torch.randn((n, 2 * (hq + hkv), d), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    before, st, pos = x.clone(), torch.cuda.current_stream().cuda_stream, list(range(n))
    w = x.stride(0)
    q, k, qo, ko = x.split([hq, hkv, hq, hkv], 1)
    sa.seg_rope_rotate(_cfg(1, hq, hkv, d), sa.make_rope(**rope), q, k, n, qo, ko, q_stride=w, k_stride=w, q_out_stride=w, k_out_stride=w, stream=st)
    assert torch.equal(ref.bits(x[:, :hq + hkv]), ref.bits(before[:, :hq + hkv]))
    _check(qo.contiguous(), q.contiguous(), pos, rope, what="q")
    _check(ko.contiguous(), k.contiguous(), pos, rope, what="k")
    y = torch.cat([before[:, :hq].reshape(-1), torch.zeros(n * hq * d, dtype=torch.bfloat16, device="cuda")]).view(2, n, hq, d)
    sa.seg_rope_rotate(_cfg(1, hq, hkv, d), sa.make_rope(**rope), y[0], None, n, y[1], None, stream=st)
    _check(y[1], before[:, :hq].contiguous(), pos, rope, what="behind it")


def test_one_tensor_alone_and_positions_from_zero():
    rope, cfg = sa.make_rope(theta=10000.0), _cfg(2, 4, 2, 64)
    x = torch.randn((10, 4, 64), device="cuda")
    y = torch.empty_like(x)
    sa.seg_rope_rotate(cfg, rope, x, None, 5, y, None, fp32=True, stream=torch.cuda.current_stream().cuda_stream)
    _check(y, x, list(range(5)) * 2, dict(theta=10000.0))
    k = torch.randn((10, 2, 64), device="cuda")
    z = torch.empty_like(k)
    sa.seg_rope_rotate(cfg, rope, None, k, 5, None, z, fp32=True, stream=torch.cuda.current_stream().cuda_stream)
    _check(z, k, list(range(5)) * 2, dict(theta=10000.0))


def test_agrees_with_the_whole_head_rotation_in_place():
    """The unscaled half layout of the whole head is what seg_rope_apply does: at most one step of bf16 apart."""
    cfg = sa.make_config(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, seg_len=512, tail_len=64, kv_policy=[1, 1], rope_theta=500000.0)
    q, k = (torch.randn((2, 301, h, 128), device="cuda").to(torch.bfloat16) for h in (8, 2))
    pos0 = torch.tensor([77, 131000], device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    st = torch.cuda.current_stream().cuda_stream
    sa.seg_rope_rotate(cfg, sa.make_rope(theta=500000.0), q, k, 301, qo, ko, pos0=pos0, stream=st)
    sa.seg_rope_apply(cfg, q, k, 301, pos0, st)
    for a, b in ((qo, q), (ko, k)):
        # both are half a step and 2^-20 of at most 2 * 6 from the same number
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * torch.maximum(a.float().abs(), b.float().abs()) + 2.0 ** -15).all()


@pytest.mark.parametrize("rope", ROPES[1:6], ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items())[:60])
def test_gradient_is_the_inverse_rotation(rope):
    """Against the formula (the transpose of the map) and against differences of the forward pass: the map is linear, so a
    central difference of <g, R x> in a direction has no truncation error, and its rounding stays below the sum of the
    elements' bounds."""
    n, hq, d = 57, 4, 64
    cfg, r = _cfg(1, hq, 1, d), sa.make_rope(**rope)
    gen = torch.Generator().manual_seed(5)
    x, g, u = (torch.randn((n, hq, d), generator=gen).cuda() for _ in range(3))
    pos = torch.randint(0, 100000, (n,), generator=gen, dtype=torch.int64).cuda()
    st = torch.cuda.current_stream().cuda_stream

    def forward(y):
        out = torch.empty_like(y)
        sa.seg_rope_rotate(cfg, r, y, None, n, out, None, pos=pos, fp32=True, stream=st)
        return out

    grad = torch.empty_like(g)
    sa.seg_rope_rotate(cfg, r, g, None, n, grad, None, pos=pos, inverse=True, fp32=True, stream=st)
    _check(grad, g, pos.cpu(), rope, inverse=True)
    slope = float(((forward(x + u).double() - forward(x - u).double()) / 2 * g.double()).sum())
    size = 2 * 2.0 ** -20 * float((g.abs() * 2 * (x.abs() + u.abs()).amax()).sum())  # |a| + |b| of x + u, x - u
    assert abs(slope - float((grad.double() * u.double()).sum())) <= size


def test_whole_turns_lose_nothing_at_far_positions():
    """Position 2^40 at one radian per position: the angle is reduced before it is rounded."""
    freq = [1.0] + [0.0] * 31
    x = torch.zeros((1, 1, 64), device="cuda")
    x[..., 0] = 1.0
    y = torch.empty_like(x)
    sa.seg_rope_rotate(_cfg(1, 1, 1, 64), sa.make_rope(theta=1.0, inv_freq=freq), x, None, 1, y, None, pos=torch.tensor([1 << 40], device="cuda"),
                       fp32=True, stream=torch.cuda.current_stream().cuda_stream)
    # 2^40 / (2 pi) turns in double: 2^-16 of a turn is lost of 2^37.3 turns at 53 bits
    assert abs(float(y[0, 0, 0]) - np.cos(2.0 ** 40)) <= 2 * np.pi * 2.0 ** -15 and abs(float(y[0, 0, 32]) - np.sin(2.0 ** 40)) <= 2 * np.pi * 2.0 ** -15
