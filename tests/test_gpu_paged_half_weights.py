"""Attention over pages in fp16: weights far below the largest are kept, as the sum that divides them keeps them."""
import math

import pytest
import torch

from tests.test_gpu_paged import _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_many_faint_keys(shared, D):
    """Two keys of 65,536 outweigh each of the others by 2^26, in blocks of keys that lie side by side; their values are zero and the
    others' are 1: the result is what the faint ones weigh together.  Enough sequences read the same pages that a
    thread block has most of a sequence.  Weights are rounded beside the largest: at 2^-26 of it to within 2^-6 when the type's
    subnormals begin 2^-29 below it or further (2^-24, and weights are taken up by 2^7 at most); the result once more."""
    from paper_2402_09633_gb300 import PagedCache
    L, page, K, n = 65536, 128, 8, 19
    k, v = torch.zeros(L, K, D, dtype=torch.float16), torch.ones(L, K, D, dtype=torch.float16)
    k[[0, 128]] = 1.0
    v[[0, 128]] = 0.0
    width = L // page + 1
    pages = L // page + n
    table = torch.arange(width - 1, dtype=torch.int32).repeat(n, 1)
    table = torch.cat([table, (L // page + torch.arange(n, dtype=torch.int32))[:, None]], 1)
    extra = torch.zeros(n * page, K, D, dtype=torch.float16)
    dk, dv = torch.cat([k, extra]).cuda(), torch.cat([v, extra]).cuda()
    dk[L:] = -1.0                                            # the one position behind them weighs 2^-52 of the largest
    q = torch.ones(n, K, D, dtype=torch.float16, device="cuda")
    cache = PagedCache(dk, dv, table.contiguous().cuda(), _i32([L + 1] * n), page)
    assert pages * page == dk.shape[0]
    got = cache.attend(q, torch.arange(n + 1, dtype=torch.int32, device="cuda"), groups=_i32([0, n]) if shared else None,
                       shared=_i32([L]) if shared else None, scale=26 * math.log(2) / D, max_q=1)
    assert cache.status() == 0
    faint = (L - 2) * 2.0 ** -26
    want = faint / (2 + faint + 2.0 ** -52)
    assert float((got.double() / want - 1).abs().max()) <= 2.0 ** -6 + 2.0 ** -11 + 2.0 ** -12
