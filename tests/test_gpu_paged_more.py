"""Caches in pages and hypotheses where single cases do not look: drawn shapes, offsets past 32 bits, values that everybody sees,
other streams, graphs that are replayed with other lengths."""
import math
import random

import pytest
import torch

from tests import paged_ref as P
from tests import sequence_ref as R
from tests.test_gpu_paged import _i32, _paged, _rand, _select, _starts, _table

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("seed", range(40))
def test_drawn_calls(seed):
    r = random.Random(seed)
    K, G, D = r.choice([1, 2, 3, 4]), r.choice([1, 2, 3, 5, 8, 16, 33]), 8 * r.randint(1, 16)
    hyps = [r.choice([0, 1, 2, r.randint(1, 40)]) for _ in range(r.randint(0, 4))]
    shared = [r.choice([0, 1, r.randint(1, 2000), 128 * r.randint(1, 8)]) for _ in hyps]
    n = max(1, sum(hyps) + r.choice([0, 0, 3]))
    nq = [r.choice([0, 1, 1, 1, r.randint(1, r.choice([2, 5, 70]))]) for _ in range(n)]
    nq[r.randrange(n)] = 1
    own = [max(q, r.choice([q, q + r.randint(0, 40), r.randint(1, 600)])) for q in nq]
    _paged(r.choice([BF16, F16]), nq, own, hyps, shared, K * G, K, D, 2 ** r.randint(4, 10), seed=seed, scale=r.choice([None, None, 0.7, -0.2]),
           max_q=r.random() < 0.6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("groups,beams,vocab,n", [(1, 2, 300001, 64), (1, 16, 140000, 33), (2, 1, 131072, 17), (1, 9, 200003, 7), (3, 5, 70001, 32)])
def test_choices_of_rows_in_many_strips(dtype, groups, beams, vocab, n):
    rows = groups * beams
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(rows, vocab, generator=g).to(dtype)
    x[torch.rand(rows, vocab, generator=g) < 0.3] = -math.inf
    _select(x, -torch.rand(rows, generator=g), beams, n)
    few = torch.randint(0, 4, (rows, vocab), generator=g).to(dtype)          # ties: the lowest places win
    few[:, :vocab // 3] = 0
    _select(few, torch.zeros(rows), beams, n)
    rare = torch.full((rows, vocab), -math.inf, dtype=dtype)                  # fewer candidates than places
    rare[:, vocab - 5:] = 1.0
    rare[0, vocab // 2] = 2.0
    _select(rare, torch.zeros(rows), beams, n)


@pytest.mark.parametrize("seed,n,groups", [(0, 800, 3), (1, 2000, 700), (2, 500, 450), (3, 1500, 0)])
def test_many_sequences(seed, n, groups):
    """More than a thread block looks at by itself, and more rows than the join has warps."""
    r = random.Random(seed)
    hyps = [r.choice([0, 1, 2, 3]) for _ in range(groups)] if groups > 3 else [r.randint(1, 200) for _ in range(groups)]
    while sum(hyps) > n:
        hyps[r.randrange(groups)] = 0
    shared = [r.choice([0, 1, r.randint(1, 150)]) for _ in hyps]
    nq = [r.choice([0, 1, 1, 2]) for _ in range(n)]
    own = [max(q, r.randint(0, 40)) for q in nq]
    _paged(r.choice([BF16, F16]), nq, own, hyps, shared, 6, 2, 64, 16, seed=seed)


@pytest.mark.parametrize("seed", range(25))
def test_drawn_choices(seed):
    r = random.Random(seed)
    groups, beams, vocab = r.randint(1, 6), r.randint(1, 64), int(math.exp(r.uniform(0, math.log(9000))))
    rows = groups * beams
    dtype = r.choice([F32, BF16, F16])
    x = _rand(rows, vocab, dtype=dtype, seed=seed, scale=r.choice([0.01, 1.0, 10.0]))
    g = torch.Generator().manual_seed(seed)
    x[torch.rand(x.shape, generator=g) < r.choice([0.0, 0.3, 0.97])] = -math.inf
    ended = torch.rand(rows, generator=g) < 0.3 if r.random() < 0.5 else None
    _select(x, -r.choice([1.0, 30.0]) * torch.rand(rows, generator=g), beams, r.randint(1, 64), ended, end=r.randint(0, vocab))


def test_values_that_everybody_sees_and_keys_that_nobody_should():
    """A NaN among the shared values makes that element of every hypothesis' result NaN, one among a hypothesis' own only its own."""
    def spoil(k, v, rows, part, length):
        v[rows(0, 17, 18), :, 5] = math.nan
        v[rows(2, 200, 201), :, 9] = math.inf
    for D in (64, 128):
        got = _paged(BF16, [1] * 5, [30, 40, 50, 60, 1], [5], [190], 4, 2, D, 16, seed=3, fill=spoil)
        bad = ~torch.isfinite(got.float())
        assert bool(bad[:, :, 5].all()) and bool(bad[2, :, 9].all())
        bad[:, :, 5] = False
        bad[2, :, 9] = False
        assert not bool(bad.any())


def test_offsets_past_32_bits():
    """Rows of a cache that lie more than 2^32 bytes from its start, written by append and read by attend and reorder."""
    from paper_2402_09633_gb300 import PagedCache, Rotary, beam_reorder
    page, K, H, D, pages = 128, 8, 8, 128, 20000                 # 5.2 GB each of keys and values
    k, v = (torch.empty(pages * page, K, D, dtype=BF16, device="cuda") for _ in range(2))
    far = [[pages - 1, 3, pages - 5], [pages - 2, 7, pages - 9]]
    table, length = _i32(far), _i32([130, 300])
    cache = PagedCache(k, v, table, length, page)
    new = _rand(430, 2 * K, D, dtype=BF16, seed=1)
    dev = new.cuda()
    cache.append(Rotary(D), _i32([0, 130, 430]), dev[:, :K], dev[:, K:])
    q = _rand(2, H, D, dtype=BF16, seed=2)
    got = cache.attend(q.cuda(), _i32([0, 1, 2]), max_q=1).cpu()
    assert cache.status() == 0
    for b, (a, z) in enumerate(((0, 130), (130, 430))):
        kk, _ = R.rotate(new[a:z, :K], torch.arange(z - a), D, "half")
        at = P.rows_of(table.cpu(), page, b, 0, z - a)
        assert torch.equal(v[at.cuda()].cpu(), new[a:z, K:])
        want, tol = R.attention(q[b:b + 1], kk.to(BF16), new[a:z, K:], R.visible(1, z - a, -1, 0, 0), 1 / math.sqrt(D))
        stored = k[at.cuda()].cpu()                              # what the keys' own rounding leaves
        want, tol = R.attention(q[b:b + 1], stored, new[a:z, K:], R.visible(1, z - a, -1, 0, 0), 1 / math.sqrt(D))
        assert bool(((got[b:b + 1].double() - want).abs() <= tol).all())
    length.copy_(_i32([300, 300]))
    beam_reorder(_i32([1, 1]), 2, caches=[cache])
    assert cache.status() == 0 and table[0].tolist() == [pages - 2, 7, pages - 5]
    assert torch.equal(v[(pages - 5) * page:(pages - 5) * page + 44], v[(pages - 9) * page:(pages - 9) * page + 44])
    states = torch.empty(4, 1 << 31, dtype=torch.uint8, device="cuda")
    states[:, -5:] = torch.arange(4, device="cuda")[:, None]
    beam_reorder(_i32([1, 0, 1, 1]), 2, [states])
    assert states[:, -1].tolist() == [1, 0, 3, 3]


def test_logits_past_2_to_the_31_elements():
    from paper_2402_09633_gb300 import beam_select
    rows, vocab, beams = 2700, 800003, 3
    x = torch.randn(1, vocab, device="cuda").to(BF16).repeat(rows, 1)
    x[-2, 5], x[-1, vocab - 1], x[7, 100] = 50.0, 60.0, 70.0
    s, p, t = beam_select(x, torch.zeros(rows, device="cuda"), beams, best=2)
    assert p[-2:].tolist() == [1, 2] and t[-2:].tolist() == [5, vocab - 1] or p[-2:].tolist() == [2, 1]
    assert (int(p[4]), int(t[4])) == (1, 100) and float(s[-2:].min()) > -1e-3


def test_fp32_is_refused_by_the_attention():
    from paper_2402_09633_gb300 import GnnError, PagedCache
    k = torch.zeros(32, 1, 64, device="cuda")
    cache = PagedCache(k, k.clone(), _i32([[0, 1]]), _i32([5]), 16)
    with pytest.raises(GnnError):
        cache.attend(torch.zeros(1, 1, 64, device="cuda"), _i32([0, 1]))
    with pytest.raises(AssertionError):
        cache.attend(torch.zeros(1, 1, 32, device="cuda"), _i32([0, 1]))
    with pytest.raises(AssertionError):
        cache.attend(torch.zeros(1, 1, 64, device="cuda"), _i32([0, 1]), groups=_i32([0, 1]))


def test_two_streams_read_one_cache():
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D, n = 32, 8, 2, 64, 24
    table, pages = _table(n, 40, seed=1)
    k, v = (_rand(pages * page, K, D, dtype=BF16, seed=s).cuda() for s in (1, 2))
    cache = PagedCache(k, v, table.cuda(), _i32([1000 + 7 * i for i in range(n)]), page)
    q = _rand(n, H, D, dtype=BF16, seed=3).cuda()
    each, groups, shared = torch.arange(n + 1, dtype=torch.int32, device="cuda"), _i32([0, n]), _i32([900])
    want = cache.attend(q, each, groups=groups, shared=shared, max_q=1)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [cache.attend(q, each, groups=groups, shared=shared, max_q=1, stream=streams[i % 3]) for i in range(30)]
    torch.cuda.synchronize()
    assert cache.status() == 0 and all(torch.equal(x, want) for x in got)


def test_a_graph_is_replayed_with_other_lengths_pages_and_groups():
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D, n = 16, 4, 2, 128, 6
    table, pages = _table(n, 30, seed=5)
    k, v = (_rand(pages * page, K, D, dtype=BF16, seed=s) for s in (1, 2))
    q = _rand(n, H, D, dtype=BF16, seed=3)
    on, length, groups, shared = table.cuda(), _i32([50] * n), _i32([0, 3, 6]), _i32([10, 20])
    cache = PagedCache(k.cuda(), v.cuda(), on, length, page)
    dq, each = q.cuda(), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache.attend(dq, each, groups=groups, shared=shared, max_q=1)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(dq, each, groups=groups, shared=shared, max_q=1)
    for lengths, cut, parts, seed in (([50] * n, [0, 3, 6], [10, 20], 5), ([480, 1, 300, 17, 16, 400], [1, 1, 4], [0, 17], 6),
                                      ([333] * n, [0, 6, 6], [333 - 1, 0], 7), ([0, 5, 0, 100, 0, 30], [0, 0, 0], [0, 0], 8)):
        t, _ = _table(n, 30, seed=seed)
        on.copy_(t)
        length.copy_(_i32(lengths))
        groups.copy_(_i32(cut))
        shared.copy_(_i32(parts))
        graph.replay()
        # sequences shorter than their group's shared part see what of it they have: through the first one's pages
        P.check_attention(out.cpu(), q, k, v, t, lengths, page, list(range(n + 1)), cut, parts, 1 / math.sqrt(D))
    assert cache.status() == 0


def test_a_graph_of_many_sequences_is_replayed_with_other_lengths():
    """Their weights are a kernel's of their own; calls that share the graph's stream write lengths right before it."""
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D, n = 16, 6, 2, 64, 900
    table, pages = _table(n, 4, seed=5)
    k, v = (_rand(pages * page, K, D, dtype=BF16, seed=s) for s in (1, 2))
    q = _rand(n, H, D, dtype=BF16, seed=3)
    length, groups, shared = _i32([50] * n), _i32([0, 300, 900]), _i32([10, 20])
    cache = PagedCache(k.cuda(), v.cuda(), table.cuda(), length, page)
    dq, each = q.cuda(), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache.attend(dq, each, groups=groups, shared=shared, max_q=1)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cache.attend(dq, each, groups=groups, shared=shared, max_q=1)
    r = random.Random(1)
    for cut, parts in (([0, 300, 900], [10, 20]), ([0, 899, 900], [33, 0]), ([5, 5, 450], [40, 17])):
        lengths = [r.randint(max(parts) + 1, 64) for _ in range(n)]
        length.copy_(_i32(lengths))
        groups.copy_(_i32(cut))
        shared.copy_(_i32(parts))
        graph.replay()
        P.check_attention(out.cpu(), q, k, v, table, lengths, page, list(range(n + 1)), cut, parts, 1 / math.sqrt(D))
    assert cache.status() == 0


def test_append_of_more_rows_than_the_offsets_say():
    from paper_2402_09633_gb300 import PagedCache, Rotary, binding
    k = _rand(64, 1, 64, dtype=F32, seed=1)
    dk, dv = k.cuda(), k.cuda()
    cache = PagedCache(dk, dv, _i32([[0, 1], [2, 3]]), _i32([20, 20]), 16)
    x = _rand(6, 1, 64, dtype=F32, seed=2).cuda()
    cache.append(Rotary(64), _i32([0, 3, 9]), x, x)              # three rows of the last sequence are not there
    assert binding.ERRORS[cache.status()] == "INDEX_RANGE"
    assert cache.append(Rotary(64), _i32([0, 0, 0]), x, x) is None and cache.status() == 0


def test_states_keep_what_lies_between_rows():
    from paper_2402_09633_gb300 import beam_reorder
    wide = torch.arange(6 * 40, dtype=torch.int16).view(6, 40)
    dev = wide.cuda()
    beam_reorder(_i32([1, 1, 0, 2, 2, 2]), 3, [dev[:, 3:24]])
    want = wide.clone()
    want[:, 3:24] = wide[[1, 1, 0, 5, 5, 5], 3:24]
    assert torch.equal(dev.cpu(), want)
    one = dev[:, 39].clone()
    got, = beam_reorder(_i32([2, 2, 2, 0, 1, 1]), 3, [one], out=[torch.empty_like(one)])
    assert torch.equal(got.cpu(), one.cpu()[[2, 2, 2, 3, 4, 4]])


def test_starts_helper():
    assert _starts([2, 0, 3]) == [0, 2, 2, 5]
