"""Attention over pages where a sequence has more queries than the call announced: it is reported, and only its own rows are undefined."""
import pytest
import torch

from tests.test_gpu_paged import _i32, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,H,K,long", [(40, 4, 2, 5), (40, 4, 2, 200), (9, 64, 1, 3), (700, 2, 1, 40)])
def test_the_other_sequences_are_computed(n, H, K, long):
    from paper_2402_09633_gb300 import PagedCache, binding
    page, D, width = 16, 64, 15
    k, v = (_rand(n * width * page, K, D, dtype=torch.bfloat16, seed=s).cuda() for s in (1, 2))
    table = torch.arange(n * width, dtype=torch.int32, device="cuda").view(n, width)
    cache = PagedCache(k, v, table, _i32([200 + i % 40 for i in range(n)]), page)
    for b in sorted({0, 7, n // 2 - 1, n // 2, n - 1}):
        nq = [1] * n
        nq[b] = long
        start = [0]
        for x in nq:
            start.append(start[-1] + x)
        q = _rand(start[-1], H, D, dtype=torch.bfloat16, seed=3).cuda()
        want = cache.attend(q, _i32(start), max_q=long)
        assert cache.status() == 0
        got = cache.attend(q, _i32(start), max_q=1)
        assert binding.ERRORS[cache.status()] == "INDEX_RANGE"
        others = torch.ones(start[-1], dtype=torch.bool)
        others[start[b]:start[b + 1]] = False
        # two results, each off by the roundings of its weights and of itself: 2^-8 of the mean magnitude of v, which lies below the largest result
        off = (got.float() - want.float())[others.cuda()].abs().max()
        assert float(off) <= 2 * (2.0 ** -8 + 2.0 ** -8) * float(want.float().abs().max())
