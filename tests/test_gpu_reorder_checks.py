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


def _two_caches(**other):
    from paper_2402_09633_gb300 import PagedCache
    page = 16
    pools = [_rand(8 * page, 1, 32, dtype=F32, seed=s) for s in range(4)]
    table, length = _i32([[0, 1], [2, 3]]), _i32([17, 17])
    dev = [x.cuda() for x in pools]
    a = dict(table=table, kv_len=length, page_size=page)
    caches = [PagedCache(dev[0], dev[1], **a), PagedCache(dev[2], dev[3], **{**a, **other})]
    return caches, dev, pools, table


@pytest.mark.parametrize("bad", ["table", "kv_len", "page_size", "beams", "generator"])
def test_nothing_moves_where_a_cache_is_refused(bad):
    from paper_2402_09633_gb300 import GnnError, beam_reorder
    other = dict(table=dict(table=_i32([[0, 1], [2, 3]])), kv_len=dict(kv_len=_i32([17, 17])), page_size=dict(page_size=32)).get(bad, {})
    caches, dev, pools, table = _two_caches(**other)
    rows, beams = (66, 66) if bad == "beams" else (2, 2)
    x = torch.arange(float(rows))
    state, out = x.cuda(), torch.zeros(rows, device="cuda")
    parents = _i32([i ^ 1 for i in range(rows)])
    if bad == "generator":                                   # taken as a list is
        beam_reorder(parents, beams, (s for s in [state]), caches=(c for c in caches))
        assert state.tolist() == [1.0, 0.0] and all(torch.equal(d[16:17].cpu(), p[48:49]) for d, p in zip(dev, pools))
        return
    for kw in (dict(), dict(out=[out])):
        with pytest.raises((GnnError, AssertionError)):
            beam_reorder(parents, beams, [state], caches=caches, **kw)
        assert torch.equal(state.cpu(), x) and not bool(out.any())
        assert all(torch.equal(d.cpu(), p) for d, p in zip(dev, pools)) and table.tolist() == [[0, 1], [2, 3]]


def test_nothing_moves_where_a_state_is_refused():
    from paper_2402_09633_gb300 import GnnError, beam_reorder
    caches, dev, pools, table = _two_caches()
    wide = torch.arange(20.0).view(2, 10).cuda()
    states = [torch.arange(2.0).cuda(), wide[:, :4]]
    parents = _i32([1, 0])
    for out in ([torch.zeros(2, device="cuda"), wide.view(-1)[:8].view(2, 4)],                 # in place, but rows elsewhere
                [torch.zeros(2, device="cuda"), torch.zeros(2, 5, device="cuda")], [torch.zeros(2, device="cuda")],
                [torch.zeros(2, device="cuda"), torch.zeros(2, 4, dtype=torch.int32, device="cuda")]):
        with pytest.raises((GnnError, AssertionError)):
            beam_reorder(parents, 2, states, out=out, caches=caches)
        assert all(torch.equal(d.cpu(), p) for d, p in zip(dev, pools)) and table.tolist() == [[0, 1], [2, 3]]
        assert not bool(out[0].any()) and torch.equal(wide.cpu(), torch.arange(20.0).view(2, 10))
    beam_reorder(parents, 2, states, caches=caches)          # and with what is right it goes through
    assert states[0].tolist() == [1.0, 0.0] and wide[0, :4].tolist() == [10.0, 11.0, 12.0, 13.0]
    assert all(torch.equal(d[16:17].cpu(), p[48:49]) for d, p in zip(dev, pools))


def test_a_cache_that_two_layers_have_is_moved_once():
    """Every slot's begun page changes places with another's: moved twice, it would be where it was."""
    from paper_2402_09633_gb300 import PagedCache, beam_reorder
    page, n = 64, 32
    table, pages = _table(n, 2, seed=3)
    k, v, more = (_rand(pages * page, 2, 64, dtype=F32, seed=s) for s in (1, 2, 3))
    parents = [i ^ 1 for i in range(n)]
    want = []
    for x in (k, v, more):
        y = x.clone()
        for i in range(n):
            a, b = int(table[i, 1]) * page, int(table[parents[i], 1]) * page
            y[a:a + 50] = x[b:b + 50]
        want.append(y)
    new = table.clone()
    new[:, 0] = table[parents, 0]
    dk, dv, dm = k.cuda(), v.cuda(), more.cuda()
    on, length = table.cuda(), _i32([page + 50] * n)
    both, tied = PagedCache(dk, dv, on, length, page), PagedCache(dm, dm, on, length, page)
    beam_reorder(_i32(parents), n, caches=[both, tied] + [both] * 20)
    assert both.status() == 0 and torch.equal(on.cpu(), new)
    assert all(torch.equal(x.cpu(), y) for x, y in zip((dk, dv, dm), want))
