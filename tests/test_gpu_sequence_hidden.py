"""New queries over a cache: values that only other queries of the sequence see may hold anything."""
import math

import pytest
import torch

from tests.test_gpu_sequence import _attend, _rand

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


# In each, some row tile (8 or 16 rows) has one query only.
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("H,K,nq", [(16, 1, 2), (32, 1, 2), (64, 2, 3), (8, 1, 3), (8, 1, 5), (16, 2, 5), (4, 1, 5),
                                    (1, 1, 17), (12, 1, 4)])
@pytest.mark.parametrize("n,left", [(70, 50), (1500, 900)])       # short ones go to tiles of 128 queries
def test_values_that_another_query_sees(n, left, H, K, nq, dtype):
    q, k, v = (_rand(r, h, 64, dtype=dtype, seed=h + r) for r, h in ((nq, H), (n, K), (n, K)))
    last, edge = v.clone(), v.clone()
    last[n - 1, 0, 5] = math.nan                             # the last query's own value
    last[n - 1, K - 1, 60] = math.inf
    got = _attend(q, k, last, [0, nq], [0], [n], -1, 0, 0, max_q=nq, max_kv=n)
    assert torch.isfinite(got[:nq - 1]).all() and not torch.isfinite(got[nq - 1]).all()
    edge[n - nq - left, 0, 5] = -math.inf                    # the first query's left edge
    edge[n - nq - left, K - 1, 60] = math.nan
    for sinks in (0, 3):
        got = _attend(q, k, edge, [0, nq], [0], [n], left, 0, sinks, max_q=nq, max_kv=n)
        assert torch.isfinite(got[1:]).all() and not torch.isfinite(got[0]).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_among_many_sequences(dtype):
    """More sequences than a block sums up the lengths of, and some in between, two queries each."""
    for seqs in (150, 1100):
        H, nq, n = 16, 2, 40
        q = _rand(seqs * nq, H, 32, dtype=dtype, seed=1)
        k, v = (_rand(seqs * n, 1, 32, dtype=dtype, seed=s) for s in (2, 3))
        v[n - 1::n, 0, 3] = math.nan
        starts = [n * b for b in range(seqs)]
        got = _attend(q, k, v, [nq * b for b in range(seqs + 1)], starts, [n] * seqs, 20, 0, 2, max_q=nq, max_kv=n)
        assert torch.isfinite(got[0::2]).all() and torch.isnan(got[1::2, :, 3]).all()
