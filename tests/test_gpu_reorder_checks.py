"""What moving hypotheses' states reports and refuses."""
import pytest
import torch

from tests.test_gpu_paged import _i32, _rand, _table

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("table,length,beams", [([[0, 1], [2, 3]], [17, 18], 2), ([[0, 1], [2, 3]], [33, 33], 2),
                                                ([[0, 1], [2, 3]], [-1, -1], 2), ([[0, 1], [2, 3]], [5, 33], 1),
                                                ([[0, 1], [2, 3]], [-7, 32], 1)])
def test_lengths_are_looked_at_where_nothing_moves(table, length, beams):
    from paper_2402_09633_gb300 import PagedCache, beam_reorder, binding
    page = 16
    k = _rand(4 * page, 1, 32, dtype=F32, seed=1)
    on, dk, dv = torch.tensor(table, dtype=torch.int32).cuda(), k.cuda(), k.cuda()
    cache = PagedCache(dk, dv, on, _i32(length), page)
    beam_reorder(_i32([i % beams for i in range(2)]), beams, caches=[cache])
    assert binding.ERRORS.get(cache.status()) == "INDEX_RANGE"
    assert torch.equal(dk.cpu(), k) and on.cpu().tolist() == table
    cache.kv_len.copy_(_i32([32, 32]))                       # as many as the table holds
    beam_reorder(_i32([i % beams for i in range(2)]), beams, caches=[cache])
    assert cache.status() == 0
