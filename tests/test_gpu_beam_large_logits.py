"""The choice of continuations among logits of any finite magnitude: masks that are large negative numbers, rows that hold nothing
else, and logits that are large themselves."""
import math

import pytest
import torch

from tests.test_gpu_paged import _rand, _select

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
MASKS = [(t, x) for t in (F32, BF16) for x in (torch.finfo(t).min, -1e9, -1e10, -1e12, -1e15, -1e20, -1e30, -1e38)] + \
    [(F16, torch.finfo(F16).min), (F16, -1e4)]
# one strip to a row, rows that start between two aligned pieces, many strips to a row
SIZES = [(1000, 4, 2), (4099, 3, 3), (20011, 4, 1)]


def _scores(rows):
    """Apart by more than a rounding of the largest values' sums, and not in order."""
    return -torch.tensor([0.75 * ((5 * i) % rows) + 0.125 for i in range(rows)])


@pytest.mark.parametrize("dtype,mask", MASKS)
@pytest.mark.parametrize("vocab,beams,groups", SIZES)
def test_masked_candidates(dtype, mask, vocab, beams, groups):
    rows = beams * groups
    for part in range(4):
        x = _rand(rows, vocab, dtype=dtype, seed=vocab + part, scale=2.0)
        if part == 0:                                        # what a lane takes first, and pieces elsewhere
            for a in (0, 16, 512, vocab // 2 // 16 * 16, vocab - 16):
                x[:, a:a + 16] = mask
        elif part == 1:                                      # a contiguous half
            x[:, :vocab // 2] = mask
            x[1, vocab // 2:] = mask
            x[1, :vocab // 2] = 0.25
        elif part == 2:                                      # all but a few here and there
            keep = torch.rand(rows, vocab, generator=torch.Generator().manual_seed(vocab)) < 60 / vocab
            keep[:, [7, vocab // 3, vocab - 1]] = True
            x = torch.where(keep, x, torch.tensor(mask, dtype=dtype))
        else:                                                # one hypothesis of each group has no other candidates
            x[::beams] = mask
        _select(x, _scores(rows), beams, 3)


@pytest.mark.parametrize("dtype,mask", MASKS)
@pytest.mark.parametrize("vocab,beams,groups", SIZES)
def test_all_but_one_and_all(dtype, mask, vocab, beams, groups):
    rows = beams * groups
    x = torch.full((rows, vocab), mask, dtype=dtype)
    _select(x, _scores(rows), beams, 7)                      # score - log(vocab) each, the lowest tokens first
    for at in (0, vocab // 2, vocab - 1):
        y = x.clone()
        y[:, at] = 0.5
        _select(y, _scores(rows), beams, beams)              # and no more: the others lie as far as the mask says
        y[0] = mask
        _select(y, _scores(rows), beams, beams)


@pytest.mark.parametrize("dtype,mask", [m for m in MASKS if m[1] <= -1e20])
def test_masked_candidates_are_chosen_where_there_are_no_others(dtype, mask):
    """Values that 64 bits do not tell apart are ties, which go to the lowest hypothesis and token."""
    x = torch.full((4, 900), mask, dtype=dtype)
    x[0, 5], x[1, 6], x[3, 899] = 1.0, 2.0, -1.0
    _select(x, torch.tensor([0.0, -1.0, -40.0, -2.0]), 4, 64)


@pytest.mark.parametrize("dtype,top", [(F32, 1e9), (F32, 3e9), (F32, 1e10), (F32, 1e20), (F32, 3e38), (F32, torch.finfo(F32).max),
                                       (BF16, 1e10), (BF16, 3e38), (BF16, torch.finfo(BF16).max), (F16, torch.finfo(F16).max)])
@pytest.mark.parametrize("vocab,beams,groups", SIZES)
def test_large_logits(dtype, top, vocab, beams, groups):
    rows = beams * groups
    x = _rand(rows, vocab, dtype=dtype, seed=vocab, scale=2.0)
    for i in range(rows):                                    # a few candidates beside which the others are nothing
        x[i, [i, vocab // 2 + 3 * i, vocab - 1 - i]] = top
    _select(x, _scores(rows), beams, 2 * beams)
    x[1] = 0.5                                               # beside a hypothesis of ordinary ones
    _select(x, _scores(rows), beams, 3)
    _select(torch.full((rows, vocab), top, dtype=dtype), _scores(rows), beams, 7)


@pytest.mark.parametrize("at", [2.0 ** 19, 2.0 ** 20, 2.0 ** 21, 3e7])
@pytest.mark.parametrize("vocab,beams", [(1000, 4), (30011, 3)])
def test_rows_about_a_large_value(at, vocab, beams):
    """A softmax does not change when all of a row's logits move, however far."""
    for sign in (-1, 1):
        x = sign * at + _rand(beams, vocab, dtype=F32, seed=vocab, scale=3.0)
        _select(x, _scores(beams), beams, 16)
        x[:, vocab // 3:] -= 40.0                            # parts of a row that weigh little
        x[0, :vocab // 3] = -math.inf
        _select(x, _scores(beams), beams, 16)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinite_and_nan_logits_among_large_ones(dtype):
    x = torch.full((6, 2000), torch.finfo(dtype).min, dtype=dtype)
    x[1, 700], x[2, 9], x[3, 1500], x[4] = math.nan, math.inf, -math.inf, -math.inf
    x[5] = torch.finfo(dtype).max
    x[5, 3] = math.inf
    _select(x, torch.zeros(6), 6, 12)                        # rows 1, 2, 4 and 5 have no continuation
    _select(x[[1, 2, 4, 5]], torch.zeros(4), 4, 3)


def test_equal_rows_tie_at_any_magnitude():
    for value in (-1e10, 1e10, 3e38, -2.0 ** 20 - 5):
        row = (value + _rand(1, 20011, dtype=F32, seed=5, scale=abs(value) / 100)).clamp(torch.finfo(F32).min, torch.finfo(F32).max)
        _select(row.repeat(8, 1), torch.full((8,), -3.7), 8, 20)
