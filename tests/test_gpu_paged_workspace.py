"""The attention's workspace follows the query rows that there are, and not how many sequences, groups or unknown lengths they are of."""
import ctypes

import pytest
import torch

from tests.test_gpu_paged import _i32, _paged, _rand, _table

pytestmark = pytest.mark.gpu


def _bytes(cache, q, n_groups, max_q):
    from paper_2402_09633_gb300 import paged as G
    from paper_2402_09633_gb300 import sequence as Q
    view = Q._fields(q, cache.dtype, cache.device, cache.dim)
    at, size = cache.kv_len.data_ptr(), ctypes.c_uint64()
    call = G._ATTEND(*view, *view, at, at if n_groups else 0, at if n_groups else 0, q.shape[0], n_groups, max_q, 0.1, 0, 0, 0)
    assert G._library().gnn_paged_workspace(cache.pages, call, ctypes.byref(size)) == 0
    return size.value


@pytest.mark.parametrize("n,rows,n_groups,max_q,H,K,D", [
    (20000, 20000, 0, 0, 16, 4, 128), (20000, 20000, 0, 1, 16, 4, 128), (20000, 20000, 0, 0, 2, 2, 64), (512, 512, 1, 0, 16, 4, 128),
    (16384, 16384, 4096, 1, 16, 4, 128), (20000, 20100, 0, 40, 2, 2, 64), (3, 4096, 2, 0, 16, 4, 128), (1, 1, 0, 0, 1, 1, 8)])
def test_bytes(n, rows, n_groups, max_q, H, K, D):
    """Two places for each row and head, as many again where there are groups, up to 256 rows for each thread block, and 8 bytes to
    an item of work: at most one to a tile's rows and one to a sequence or group, for each key head."""
    from paper_2402_09633_gb300 import PagedCache
    k = torch.zeros(32, K, D, dtype=torch.bfloat16, device="cuda")
    cache = PagedCache(k, k, torch.zeros(n, 2, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda"), 16)
    q = torch.zeros(rows, H, D, dtype=torch.bfloat16, device="cuda")
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    kinds = 2 if n_groups else 1
    place = kinds * (2 * rows * H + 256 * sms) * (D + 2) * 4
    items = 8 * K * (n + n_groups + 2 * (rows * (H // K) // 64 + 1)) + 8 * (n + n_groups)
    assert _bytes(cache, q, n_groups, max_q) <= place + items + 4096


@pytest.mark.parametrize("known", [False, True])
def test_many_short_sequences(known):
    n = 6000
    _paged(torch.float16, [1] * n, [1 + (5 * i) % 37 for i in range(n)], [2, 4000, 1], [200, 40, 3], 4, 2, 64, 16, seed=5, max_q=known)


@pytest.mark.parametrize("known", [False, True])
def test_ragged_queries(known):
    """Sequences of a few and of many new rows, in packs and in tiles."""
    for most, n in ((3, 500), (40, 90), (300, 20)):
        nq = [(7 * i) % most + (i % 3 > 0) for i in range(n)]
        own = [x + (11 * i) % 200 for i, x in enumerate(nq)]
        _paged(torch.bfloat16, nq, own, [n // 2, n // 4], [333, 50], 6, 2, 64, 16, seed=most, max_q=known)


@pytest.mark.parametrize("n", [5, 33, 45])
@pytest.mark.parametrize("max_q", [0, 2])
def test_rows_around_the_sequences(n, max_q):
    """Rows before the first and behind the last sequence, in packs that are not full: they are left as they were."""
    import math

    from paper_2402_09633_gb300 import PagedCache
    from tests import paged_ref as P
    page, H, K, D = 16, 4, 2, 64
    nq = [1 + i % 2 for i in range(n)]
    start = [7]
    for x in nq:
        start.append(start[-1] + x)
    length = [20 + (9 * i) % 60 for i in range(n)]
    table, pages = _table(n, 5, seed=n)
    q = _rand(start[-1] + 100, H, D, dtype=torch.float16, seed=1)
    k, v = (_rand(pages * page, K, D, dtype=torch.float16, seed=s) for s in (2, 3))
    cache = PagedCache(k.cuda(), v.cuda(), table.cuda(), _i32(length), page)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    got = cache.attend(q.cuda(), _i32(start), groups=_i32([1, n]), shared=_i32([16]), max_q=max_q, out=out).cpu()
    assert cache.status() == 0
    first = table.clone()
    first[1:, 0] = table[1, 0]
    P.check_attention(got, q, k, v, first, length, page, start, [0], [], 1 / math.sqrt(D))
    assert bool((got[:7] == 7).all()) and bool((got[start[-1]:] == 7).all())
