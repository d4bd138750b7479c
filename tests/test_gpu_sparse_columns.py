"""Attention over chosen blocks, chunks: what a token gets depends on its own rows, list and queries, not on the tokens whose columns lie beside its
own -- and so not on which ones those are, which for listed blocks the order of atomics decides."""
import pytest
import torch

from paged_ref import Pool
from test_gpu_sparse import BF16, _attend, _lists

pytestmark = pytest.mark.gpu

# Keys of four times the usual magnitude: from one tile of 32 rows to the next some columns' largest scores grow by more than 2^8, their neighbours'
# by less.  Listed blocks are taken once for all tokens and windows cut into shares (test_chosen_forms.py): d, g, 8-bit rows, tokens, blocks
CHUNKS = [(128, 4, False, 1400, 16), (128, 4, True, 2600, 16), (64, 1, False, 1400, 16)]
HELD, BLOCK, SEG, TAIL, POLICY = 700, 64, 1000, 300, [2, 1]


@pytest.mark.parametrize("out_fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("d,g,e4m3,n,chosen", CHUNKS)
def test_a_column_does_not_depend_on_its_neighbours(d, g, e4m3, n, chosen, out_fp32):
    pool = Pool(batch=1, hkv=2, d=d, page_rows=BLOCK, max_pages=-(-(HELD + n) // BLOCK), e4m3=e4m3).fill([HELD + n])
    if e4m3:
        pool.k_scale += 2
    else:
        pool.k *= 4
    q = torch.randn((n, 2 * g, d), generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    lists = _lists(pool, [n], chosen, BLOCK, POLICY)
    kw = dict(hq=2 * g, policy=POLICY, seg=SEG, tail=TAIL, out_fp32=out_fp32)
    out, lse, odd = _attend(pool, BLOCK, [n], chosen, q=q, lists=lists, **kw)
    assert not odd.any()
    # every other token has other queries and another list
    others = q.clone()
    others[1::2] = 2 * torch.randn((n // 2, 2 * g, d), generator=torch.Generator().manual_seed(2)).to(BF16).cuda()
    changed = lists.clone()
    changed[1::2] = _lists(pool, [n], chosen, BLOCK, POLICY, seed=5)[1::2]
    again, lse_again, _ = _attend(pool, BLOCK, [n], chosen, q=others, lists=changed, **kw)
    for h, name in ((0, "listed blocks"), (1, "window")):
        heads = slice(h * g, (h + 1) * g)
        assert not torch.equal(out[1::2, heads], again[1::2, heads])
        for what, x, y in (("out", out, again), ("lse", lse, lse_again)):
            differs = int((x[::2, heads] != y[::2, heads]).sum())
            assert differs == 0, f"{name}: {differs} numbers of {what} depend on other tokens"
