"""Packed attention where scores outgrow, within one block of keys, everything that the block before held."""
import math

import pytest
import torch

from tests.test_gpu_sequence import _attend, _rand

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

# Runs of keys and their scores in powers of two; blocks are 128 keys.  The first five: sums beyond 2^128 of weights
# below it, and sums that a later block has to bring down by 2^126 and more in two steps.
JUMPS = [
    [(254, 0), (2, 127.5)],
    [(252, 0), (4, 126)],
    [(192, 0), (64, 122)],
    [(128, 0), (128, 122), (64, 122)],
    [(128, 0), (128, 120), (1, 127), (127, 0)],
    [(128, 0), (128, 60), (128, 100), (70, 64)],
    [(128, 0), (128, 100), (128, 0), (1, 227), (60, 3)],
    [(128, -90), (128, 60), (128, 180), (128, 179)],
    [(128, 0), (128, 200), (5, 255)],
    [(128, 0), (128, 9), (128, 18), (128, 12)],
    [(128, 250), (128, 0), (128, 120), (128, 246)],
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("left,right,sinks", [(-1, -1, 0), (-1, 0, 0), (200, 60, 5)])
@pytest.mark.parametrize("case", range(len(JUMPS)))
def test_scores_that_jump(case, left, right, sinks, D, dtype):
    scores = torch.tensor([float(s) for n, s in JUMPS[case] for _ in range(n)])
    n = scores.numel()
    q, k = torch.zeros(2, n, 1, D, dtype=dtype)
    q[:, 0, 0] = 1
    k[:, 0, 0] = scores.to(dtype)
    assert torch.equal(k[:, 0, 0].float(), scores)
    v = _rand(n, 1, D, dtype=dtype, seed=case, scale=0.5)
    _attend(q, k, v, [0, n], None, None, left, right, sinks, scale=math.log(2.0))


def test_a_sum_beyond_fp32_of_equal_weights():
    n, D = 256, 64
    q = torch.full((n, 1, D), 3.25, dtype=BF16)
    k, v = q.clone(), torch.full((n, 1, D), 0.25, dtype=BF16)
    k[:128] = 0
    got = _attend(q, k, v, [0, n], None, None, -1, -1, 0)
    assert bool((got == 0.25).all())
