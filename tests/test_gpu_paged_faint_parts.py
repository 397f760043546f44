"""Attention over pages: a value that is not finite and that a query sees makes its result not finite, however little its key weighs
and wherever the work is cut."""
import math

import pytest
import torch

from tests.test_gpu_paged import _i32, _rand, _starts, _table

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def _run(dtype, nq, length, spoil, groups=None, shared=None, D=64, K=2, G=2, page=32, max_q=0, loud=(0, 5)):
    """Keys without weight beside one of sequence loud[0] at position loud[1] (and shared by all, if that is), whose score is some 500
    above theirs; spoil(k, v, rows) puts in what is not finite."""
    from paper_2402_09633_gb300 import PagedCache
    n = len(nq)
    table, pages = _table(n, -(-max(length) // page), seed=3)
    k = torch.zeros(pages * page, K, D, dtype=dtype)
    v = _rand(pages * page, K, D, dtype=dtype, seed=4)

    def rows(b, a, z):
        j = torch.arange(a, z)
        return table[b].long()[j // page] * page + j % page
    for b in range(n):
        at = loud[1] if b == loud[0] or shared is None else 0
        if shared is None or b == loud[0]:
            k[rows(b, at, at + 1)] = 8.0
    spoil(k, v, rows)
    cache = PagedCache(k.cuda(), v.cuda(), table.cuda(), _i32(length), page)
    q = torch.full((sum(nq), K * G, D), 8.0, dtype=dtype)
    got = cache.attend(q.cuda(), _i32(_starts(nq)), groups=None if groups is None else _i32(groups),
                       shared=None if shared is None else _i32(shared), max_q=max_q)
    assert cache.status() == 0
    return torch.isfinite(got.float()).cpu()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [5, 130, 4000, 19990])
def test_own_keys(dtype, value, at):
    def spoil(k, v, rows):
        v[rows(0, at, at + 1), 1, 9] = value
    fine = _run(dtype, [1, 1], [20000, 300], spoil)
    want = torch.ones(2, 4, 64, dtype=torch.bool)
    want[0, 2:, 9] = False                                   # the query heads that read key head 1
    assert torch.equal(fine, want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [40, 2500, 7999])
@pytest.mark.parametrize("hyps", [3, 40])
def test_shared_keys(D, at, hyps):
    def spoil(k, v, rows):
        v[rows(0, at, at + 1), 0, 17] = math.inf
    fine = _run(BF16, [1] * hyps, [8000 + 1 + i % 7 for i in range(hyps)], spoil, groups=[0, hyps], shared=[8000], D=D, page=128,
                max_q=1)
    want = torch.ones(hyps, 4, D, dtype=torch.bool)
    want[:, :2, 17] = False
    assert torch.equal(fine, want)


def test_new_rows_see_their_own_only():
    """The last of three new rows, behind a long cache: its value is infinite, and the first two do not see it."""
    def spoil(k, v, rows):
        v[rows(0, 15002, 15003), :, 3] = math.inf
        v[rows(1, 700, 701), :, 8] = math.nan
    for max_q in (0, 3):
        fine = _run(BF16, [3, 3, 1], [15003, 800, 90], spoil, max_q=max_q)
        want = torch.ones(7, 4, 64, dtype=torch.bool)
        want[2, :, 3] = False
        want[3:6, :, 8] = False
        assert torch.equal(fine, want)


def test_keys_whose_scores_are_minus_infinity():
    def spoil(k, v, rows):
        k[rows(0, 8000, 12000)] = -math.inf
        v[rows(0, 9000, 9001), 0, 4] = math.nan
        k[rows(1, 0, 500)] = -math.inf                       # a query all of whose scores are: zeros
        v[rows(1, 77, 78)] = math.inf
    fine = _run(BF16, [1, 1], [16000, 500], spoil)
    want = torch.ones(2, 4, 64, dtype=torch.bool)
    want[0, :2, 4] = False
    assert torch.equal(fine, want)
