"""What putting new rows in their pages reports: offsets and lengths that are out of range, of any sequence."""
import pytest
import torch

from tests.test_gpu_paged import _i32, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("start,length", [
    ([-2, 1, 2, 4], [20, 20, 20]),                           # before the first row
    ([0, 3, 2, 4], [20, 20, 20]),                            # falling
    ([2, 0, 0, 4], [20, 20, 20]),
    ([0, 1, 2, 9], [20, 20, 20]),                            # past the last row
    ([0, 1, 9, 9], [20, 20, 20]),
    ([0, 1, 2, 4], [20, -3, 20]),
    ([0, 1, 1, 4], [20, -3, 20]),                            # of a sequence without new rows
    ([0, 1, 1, 4], [20, 33, 20]),
    ([0, 1, 2, 4], [20, 40, 20])])
def test_offsets_and_lengths_out_of_range(start, length):
    from paper_2402_09633_gb300 import PagedCache, Rotary, binding
    k = _rand(6 * 16, 1, 64, dtype=torch.float32, seed=1)
    x = _rand(4, 1, 64, dtype=torch.float32, seed=2).cuda()
    cache = PagedCache(k.cuda(), k.cuda(), _i32([[0, 1], [2, 3], [4, 5]]), _i32(length), 16)
    cache.append(Rotary(64), _i32(start), x, x)
    assert binding.ERRORS.get(cache.status()) == "INDEX_RANGE"
    cache.kv_len.copy_(_i32([20, 0, 32]))                    # what is in range: none, some and all positions in use
    cache.append(Rotary(64), _i32([1, 1, 1, 3]), x, x)
    assert cache.status() == 0


def test_many_sequences_few_rows():
    from paper_2402_09633_gb300 import PagedCache, Rotary, binding
    n = 50001
    k = torch.zeros(16, 1, 64, device="cuda")
    x = _rand(1, 1, 64, dtype=torch.float32, seed=2).cuda()
    length = torch.ones(n, dtype=torch.int32, device="cuda")
    cache = PagedCache(k, k.clone(), torch.zeros(n, 1, dtype=torch.int32, device="cuda"), length, 16)
    start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    start[n // 2:] = 1
    cache.append(Rotary(64), start, x, x)
    assert cache.status() == 0
    for b in (0, 777, n // 2, n - 1):
        length[b] = -1
        cache.append(Rotary(64), start, x, x)
        assert binding.ERRORS.get(cache.status()) == "INDEX_RANGE"
        length[b] = 1
