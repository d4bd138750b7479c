"""Bounds of blocks whose keys are of very different magnitudes."""
import pytest
import torch

import sparse_ref as sref
from paged_ref import Pool
from test_gpu_sparse import BF16, _summarize

pytestmark = pytest.mark.gpu


def test_bounds_of_keys_far_below_the_largest_are_rounded_away_from_zero():
    """However small a key is beside the block's largest: an upper bound of a positive one is 1 or more, a lower bound of a negative one -1 or less
    (the quotients leave the range of 32-bit floats; the oracle's are in 64 bits)."""
    pool = Pool(batch=1, hkv=1, d=64, page_rows=16, max_pages=4).fill([64])
    blocks = sref.Blocks(pool, 16)
    for j, (large, small) in enumerate([(3.0e38, 2.0 ** -40), (3.0e38, 2.0 ** -133), (2.0 ** 40, 2.0 ** -126), (1.0e30, 2.0 ** -60)]):
        x = torch.zeros((16, 64), dtype=torch.float64)
        x[3, 0] = large
        x[:, 1] = small          # above zero in all rows
        x[:, 2] = -small         # below
        x[5, 3], x[6, 3] = small, -small
        x[7, 4] = small          # beside zeros
        x[8, 5] = -small
        page, hh, r = pool.place(0, 0, range(16 * j, 16 * j + 16))
        pool.k[page.cuda(), hh, r.cuda()] = x.to(BF16).cuda()
        want = sref.bounds_of(x.to(BF16).to(torch.float64))
        assert want[0][:6].tolist()[1:] == [1, 0, 1, 1, 0] and want[1][:6].tolist()[1:] == [0, -1, -1, 0, -1]
    _summarize(pool, blocks, None, 64, [2])
