"""Caches in pages, attention that reads shared keys once, the choice of continuations and moving states, on the GPU
against plain statements in 64 bits, at the sizes, layouts and masks where they can go wrong."""
import math

import pytest
import torch

from tests import paged_ref as P
from tests import sequence_ref as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _rand(*size, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*size, generator=g) * scale).to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


def _table(n, width, seed, spare=3):
    """Every sequence's pages, anywhere among a few more than there are."""
    p = torch.randperm(n * width + spare, generator=torch.Generator().manual_seed(seed))
    return p[:n * width].view(n, width).int().contiguous(), n * width + spare


# ------------------------------------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("new,old,heads,kv,dim,rot,page", [
    ([1], [0], 1, 1, 2, 2, 16),
    ([1, 1, 1, 1], [15, 16, 17, 300], 16, 4, 128, 128, 16),
    ([5, 0, 1, 130, 33], [3, 8, 0, 70, 31], 6, 2, 96, 40, 32),
    ([0, 0, 77], [1, 2, 51], 3, 1, 250, 30, 64),
    ([700], [1], 2, 2, 64, 64, 1024)])
def test_append(dtype, layout, normed, new, old, heads, kv, dim, rot, page):
    from paper_2402_09633_gb300 import PagedCache, Rotary
    rows, n = sum(new), len(new)
    length = [a + b for a, b in zip(new, old)]
    table, pages = _table(n, -(-max(length) // page), seed=rows)
    qkv = _rand(rows, heads + 2 * kv, dim, dtype=dtype, seed=rows + dim, scale=2.0)
    kc, vc = (_rand(pages * page, kv, dim, dtype=dtype, seed=s) for s in (8, 9))
    gq, gk = (1 + _rand(dim, dtype=F32, seed=s, scale=0.3) for s in (1, 2)) if normed else (None, None)
    cu = lambda x: None if x is None else x.cuda()           # noqa: E731
    dev, dk, dv = qkv.cuda(), kc.cuda(), vc.cuda()
    cache = PagedCache(dk, dv, table.cuda(), _i32(length), page)
    got = cache.append(Rotary(rot, layout=layout), _i32(_starts(new)), dev[:, heads:heads + kv], dev[:, heads + kv:],
                       q=dev[:, :heads], q_gain=cu(gq), k_gain=cu(gk), eps=1e-5 if normed else None)
    assert cache.status() == 0
    pos = torch.cat([torch.arange(a, a + b) for a, b in zip(old, new)])
    at = torch.cat([P.rows_of(table, page, b, old[b], length[b]) for b in range(n)])
    norm = (lambda x, g: R.norm(x, g, 1e-5)) if normed else (lambda x, g: x)
    R.check_rotated(got, *R.rotate(norm(qkv[:, :heads], gq), pos, rot, layout), normed=normed)
    R.check_rotated(dk.cpu()[at], *R.rotate(norm(qkv[:, heads:heads + kv], gk), pos, rot, layout), normed=normed)
    assert torch.equal(dv.cpu()[at], qkv[:, heads + kv:])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[at] = False
    assert torch.equal(dk.cpu()[rest], kc[rest]) and torch.equal(dv.cpu()[rest], vc[rest])


def test_append_views_positions_in_place_and_without_queries():
    from paper_2402_09633_gb300 import PagedCache, Rotary
    page, n, kv, dim = 16, 40, 3, 64
    table, pages = _table(2, 4, seed=0)
    wide = _rand(pages * page, 2 * kv, dim, dtype=BF16, seed=1)
    both = wide.cuda()                                       # keys and values side by side in a row
    start = [3, 20, 37]                                      # rows before the first and from the last on are no sequence's
    length = [17, 30]
    x = _rand(n, 2 * kv, dim, dtype=BF16, seed=2)
    dev = x.cuda()
    phi = _rand(n, dtype=F32, seed=3, scale=30.0)
    cache = PagedCache(both[:, :kv], both[:, kv:], table.cuda(), _i32(length), page)
    assert cache.append(Rotary(32), _i32(start), dev[:, :kv], dev[:, kv:], positions=phi.cuda()) is None
    at = torch.cat([P.rows_of(table, page, 0, 0, 17), P.rows_of(table, page, 1, 13, 30)])
    R.check_rotated(both.cpu()[at][:, :kv], *R.rotate(x[3:37, :kv], phi[3:37], 32, "half"), normed=False)
    assert torch.equal(both.cpu()[at][:, kv:], x[3:37, kv:])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[at] = False
    assert torch.equal(both.cpu()[rest], wide[rest])
    # queries in place; those of no sequence stay as they are
    q = _rand(n, 5, dim, dtype=BF16, seed=4)
    dq = q.cuda()
    assert cache.append(Rotary(32), _i32(start), dev[:, :kv], dev[:, kv:], q=dq, q_out=dq) is dq
    pos = torch.cat([torch.arange(17), torch.arange(13, 30)])
    R.check_rotated(dq[3:37].cpu(), *R.rotate(q[3:37], pos, 32, "half"), normed=False)
    assert torch.equal(dq.cpu()[:3], q[:3]) and torch.equal(dq.cpu()[37:], q[37:])
    assert cache.status() == 0


def test_append_leaves_bad_places_alone():
    from paper_2402_09633_gb300 import GnnError, PagedCache, Rotary, binding
    page, kv, dim = 16, 1, 64
    k0, v0 = (_rand(4 * page, kv, dim, dtype=F32, seed=s) for s in (1, 2))
    table = torch.tensor([[0, 7], [1, -1], [2, 3]], dtype=torch.int32)
    k, v = _rand(6, kv, dim, dtype=F32, seed=3).cuda(), _rand(6, kv, dim, dtype=F32, seed=4).cuda()
    for length, written in (([17, 17, 18], [3 * page, 3 * page + 1]),          # pages 7 and -1 are none
                            ([2, 33, 1], [0, 1, 2 * page])):                   # past the table; fewer positions than rows
        dk, dv = k0.cuda(), v0.cuda()
        cache = PagedCache(dk, dv, table.cuda(), _i32(length), page)
        cache.append(Rotary(64), _i32([0, 2, 4, 6]), k, v)
        assert binding.ERRORS[cache.status()] == "INDEX_RANGE" and cache.status() == 0
        changed = (dv.cpu() != v0).flatten(1).any(1).nonzero().flatten().tolist()
        # of the rows that fall on a good page: position 16 of a sequence lies on page 1 of its row
        assert set(changed) <= set(written) | {15, page + 15}
        assert set(written) <= set(changed)
    with pytest.raises(GnnError):
        cache.append(Rotary(128), _i32([0, 2, 4, 6]), k, v)


# ------------------------------------------------------------------------------------------- attention

def _paged(dtype, nq, own, hyps, shared, H, K, D, page, seed, scale=None, scale_of=1.0, garbage=math.nan, max_q=True, grouped=True,
           fill=None):
    """One call and its check.  hyps: sequences of each group (the last one's may be of none); own: positions of each sequence
    behind its group's shared ones."""
    from paper_2402_09633_gb300 import PagedCache
    n = len(nq)
    group_start = _starts(hyps)
    part = [0] * n
    for g, s in enumerate(shared):
        part[group_start[g]:group_start[g + 1]] = [s] * hyps[g]
    length = [a + b for a, b in zip(part, own)]
    table, pages = _table(n, max(1, -(-max(length) // page)), seed=seed)
    q = _rand(sum(nq), H, D, dtype=dtype, seed=seed, scale=scale_of)
    k, v = (_rand(pages * page, K, D, dtype=dtype, seed=seed + s) for s in (50, 90))
    if fill:
        fill(k, v, lambda b, a, z: P.rows_of(table, page, b, a, z), part, length)
    if garbage is not None:                                  # what no position of anybody lies in counts for nothing
        used = torch.zeros(pages * page, dtype=torch.bool)
        for b in range(n):
            used[P.rows_of(table, page, b, part[b], length[b])] = True
        for g in range(len(shared)):
            if hyps[g]:
                used[P.rows_of(table, page, group_start[g], 0, shared[g])] = True
        k[~used], v[~used] = garbage, garbage
    start = _starts(nq)
    cache = PagedCache(k.cuda(), v.cuda(), table.cuda(), _i32(length), page)
    got = cache.attend(q.cuda(), _i32(start), groups=_i32(group_start) if grouped and shared else None,
                       shared=_i32(shared) if grouped and shared else None, scale=scale, max_q=max(nq) if max_q else 0)
    again = cache.attend(q.cuda(), _i32(start), groups=_i32(group_start) if grouped and shared else None,
                         shared=_i32(shared) if grouped and shared else None, scale=scale, max_q=max(nq) if max_q else 0)
    assert cache.status() == 0
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))
    P.check_attention(got.cpu(), q, k, v, table, length, page, start, group_start, shared, 1 / math.sqrt(D) if scale is None else scale)
    return got.cpu()


PAGED = [  # new rows, own positions, sequences of each group, shared positions, heads, kv heads, dim, page
    ([1], [1], [], [], 1, 1, 64, 16),
    ([1], [0], [], [], 2, 1, 64, 16),                                # no key at all
    ([1, 1], [0, 3], [], [], 4, 2, 128, 16),
    ([1], [1], [1], [1], 1, 1, 128, 16),
    ([1, 1, 1], [1, 2, 3], [3], [127], 4, 2, 64, 16),
    ([1, 1, 1], [1, 130, 3], [3], [128], 4, 4, 128, 32),
    ([1, 1, 1], [129, 128, 127], [3], [129], 4, 1, 128, 128),
    ([1] * 5, [1, 7, 33, 2, 300], [2, 0, 3], [200, 50, 0], 6, 2, 96, 32),
    ([3] * 7, [3, 4, 5, 100, 3, 17, 200], [3, 2], [1000, 517], 6, 2, 72, 64),    # the last two are of no group
    ([2, 1, 0, 5], [2, 9, 4, 140], [4], [333], 5, 5, 40, 16),
    ([1] * 33, list(range(1, 34)), [33], [2000], 16, 4, 128, 64),
    ([1] * 100, [3] * 100, [100], [300], 8, 2, 64, 128),             # 400 rows to a key head
    ([1] * 70, [1 + i % 40 for i in range(70)], [70], [5000], 16, 4, 128, 1024),
    ([1] * 9, [17, 333, 1024, 1, 2, 900, 31, 32, 33], [], [], 12, 3, 40, 16),
    ([1], [20001], [], [], 8, 8, 8, 16),
    ([2, 2], [9000, 8000], [], [], 32, 2, 128, 256),
    ([200, 1], [300, 600], [2], [77], 4, 2, 64, 32),                 # a chunk of a prompt beside a step
    ([1, 1], [5, 6], [2], [3000], 128, 1, 32, 64),                   # all heads read one key head
    ([4, 4], [10, 40], [2], [700], 50, 2, 16, 16),                   # 25 heads to a key head: five queries to a tile
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("known", [False, True])
@pytest.mark.parametrize("case", range(len(PAGED)))
def test_attend(case, known, dtype):
    nq, own, hyps, shared, H, K, D, page = PAGED[case]
    _paged(dtype, nq, own, hyps, shared, H, K, D, page, seed=case, max_q=known)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attend_scales(dtype, scale):
    _paged(dtype, [1, 2, 1], [5, 200, 30], [2], [400], 4, 2, 64, 32, seed=5, scale=scale, scale_of=2.0)
    _paged(dtype, [1, 2, 1], [5, 200, 30], [2], [400], 4, 2, 128, 32, seed=6, scale=scale, scale_of=2.0)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_scores_that_jump(dtype, dim):
    """Keys that grow along the sequence: each block of keys outweighs all before it, and the shared part the own or the reverse."""
    def grow(k, v, rows, part, length):
        for b in range(len(length)):
            for a in range(0, length[b], 64):
                z = min(length[b], a + 64)
                k[rows(b, a, z)] *= 0.02 * (1 + a / 16)
        k.clamp_(-200, 200)
    _paged(dtype, [1] * 6, [300, 1, 64, 20, 5, 100], [4], [1500], 4, 2, dim, 64, seed=7, fill=grow, scale_of=1.5)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_hidden_values_that_are_not_finite(dtype):
    """The last of three new rows holds NaN and infinities: the first two do not see it, the third does."""
    def spoil(k, v, rows, part, length):
        at = rows(1, length[1] - 1, length[1])
        v[at], k[at] = math.nan, 1.0
        v[rows(2, length[2] - 1, length[2])] = math.inf
    got = _paged(dtype, [3, 3, 3], [40, 50, 150], [3], [300], 4, 2, 64, 16, seed=9, fill=spoil)
    assert bool(torch.isfinite(got[3:5]).all()) and not bool(torch.isfinite(got[5]).any())
    assert bool(torch.isfinite(got[6:8]).all()) and not bool(torch.isfinite(got[8]).any())


def test_attend_shared_keys_are_read_through_the_first_sequence():
    """The other sequences' entries for shared pages may be anything, and so may entries behind the last position."""
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D, S = 16, 4, 2, 64, 100
    own = [5, 30, 1]
    table, pages = _table(3, 10, seed=2)
    q = _rand(3, H, D, dtype=BF16, seed=1)
    k, v = (_rand(pages * page, K, D, dtype=BF16, seed=s) for s in (2, 3))
    length = [S + n for n in own]
    given = table.clone()
    for b in range(3):
        given[b, -(-length[b] // page):] = -5
        if b:
            given[b, :S // page] = 10 ** 9
    cache = PagedCache(k.cuda(), v.cuda(), given.cuda(), _i32(length), page)
    got = cache.attend(q.cuda(), _i32([0, 1, 2, 3]), groups=_i32([0, 3]), shared=_i32([S]))
    assert cache.status() == 0
    P.check_attention(got.cpu(), q, k, v, table, length, page, [0, 1, 2, 3], [0, 3], [S], 1 / math.sqrt(D))


def test_attend_queries_below_the_shared_length():
    """Sequences some of whose queries stand among the shared positions, or that are empty, beside ordinary ones."""
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D, S = 32, 4, 2, 128, 300
    nq, length = [1, 4, 1, 1, 2], [320, 302, 0, 120, 301]
    table, pages = _table(5, 11, seed=3)
    q = _rand(sum(nq), H, D, dtype=F16, seed=1)
    k, v = (_rand(pages * page, K, D, dtype=F16, seed=s) for s in (2, 3))
    for b in range(1, 5):                                    # the page that the shared positions end in
        frm, to = P.rows_of(table, page, 0, S // page * page, S), P.rows_of(table, page, b, S // page * page, S)
        k[to], v[to] = k[frm], v[frm]
    start = _starts(nq)
    cache = PagedCache(k.cuda(), v.cuda(), table.cuda(), _i32(length), page)
    got = cache.attend(q.cuda(), _i32(start), groups=_i32([0, 5]), shared=_i32([S])).cpu()
    assert cache.status() == 0
    P.check_attention(got, q, k, v, table, length, page, start, [0, 5], [S], 1 / math.sqrt(D))
    assert not bool(got[start[2]].any())


def test_attend_views_and_rows_of_no_sequence():
    from paper_2402_09633_gb300 import PagedCache
    page, H, K, D = 16, 6, 3, 64
    table, pages = _table(2, 20, seed=4)
    both = _rand(pages * page, 2 * K, D, dtype=BF16, seed=5)
    dev = both.cuda()
    q = _rand(H, 9, D, dtype=BF16, seed=6)                   # heads first
    out = torch.full((9, H, D + 8), 7.0, dtype=BF16, device="cuda")
    wide = torch.zeros(2, 25, dtype=torch.int32)
    wide[:, :20] = table
    cache = PagedCache(dev[:, :K], dev[:, K:], wide.cuda()[:, :20], _i32([250, 311]), page)
    got = cache.attend(q.cuda().transpose(0, 1), _i32([2, 5, 7]), groups=_i32([0, 2]), shared=_i32([240]), out=out[:, :, :D])
    assert got.data_ptr() == out.data_ptr() and cache.status() == 0
    P.check_attention(got.cpu(), q.transpose(0, 1), both[:, :K], both[:, K:], table, [250, 311], page, [2, 5, 7], [0, 2], [240],
                      1 / math.sqrt(D))
    left = out.cpu()
    assert bool((left[:2] == 7).all() and (left[7:] == 7).all() and (left[:, :, D:] == 7).all())


def test_attend_reports_what_is_out_of_range():
    from paper_2402_09633_gb300 import PagedCache, binding
    page, K, D = 16, 1, 64
    k = _rand(4 * page, K, D, dtype=BF16, seed=1).cuda()
    q = _rand(2, 2, D, dtype=BF16, seed=2).cuda()
    good = dict(table=[[0, 1], [2, 3]], length=[20, 30], start=[0, 1, 2], groups=None, shared=None, max_q=0)
    for bad in (dict(table=[[0, 4], [2, 3]]), dict(table=[[0, 1], [-1, 3]]), dict(length=[20, 33]), dict(length=[-1, 30]),
                dict(start=[0, 1, 3]), dict(start=[-1, 1, 2]), dict(groups=[0, 2], shared=[40]), dict(groups=[0, 2], shared=[-1]),
                dict(start=[0, 2, 2], max_q=1), {}):
        a = {**good, **bad}
        cache = PagedCache(k, k, torch.tensor(a["table"], dtype=torch.int32).cuda(), _i32(a["length"]), page)
        cache.attend(q, _i32(a["start"]), groups=a["groups"] and _i32(a["groups"]), shared=a["shared"] and _i32(a["shared"]),
                     max_q=a["max_q"])
        code = cache.status()
        assert binding.ERRORS.get(code, code) == ("INDEX_RANGE" if bad else 0), bad
        assert cache.status() == 0


def test_attend_many_sequences():
    n = 3000
    _paged(BF16, [1] * n, [1 + (7 * i) % 23 for i in range(n)], [1000, 0, 1500], [333, 10, 90], 2, 1, 32, 16, seed=11)


# ------------------------------------------------------------------------------------------- the choice

def _select(x, scores, beams, n, ended=None, end=0, exact=True):
    from paper_2402_09633_gb300 import beam_select
    got = beam_select(x.cuda(), scores.cuda(), beams, best=n, ended=None if ended is None else ended.cuda(), end=end)
    want = P.best(x, scores, beams, n, ended, end)
    groups = x.shape[0] // beams
    s, p, t = (a.cpu().view(groups, n) for a in got)
    same = torch.isfinite(want[0])
    assert torch.equal(torch.isfinite(s), same) and bool((s[~same] == want[0][~same]).all())
    off = ((s.double() - want[0]).abs() / P.value_error(want[0], x.shape[1]))[same]
    assert off.numel() == 0 or float(off.max()) <= 1
    assert torch.equal(p.long(), want[1]) and torch.equal(t.long(), want[2])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("groups,beams,vocab,n", [
    (1, 1, 1, 1), (1, 4, 1000, 4), (3, 1, 10, 64), (2, 3, 7, 5), (5, 8, 32003, 8), (1, 64, 517, 64), (2, 2, 100001, 33),
    (1, 5, 65536, 1), (9, 7, 4097, 7), (70, 4, 257, 4)])
def test_select(dtype, groups, beams, vocab, n):
    rows = groups * beams
    x = _rand(rows, vocab, dtype=dtype, seed=rows + vocab, scale=2.0)
    scores = -20.0 * torch.rand(rows, generator=torch.Generator().manual_seed(vocab))
    _select(x, scores, beams, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_select_ended_hidden_and_dead(dtype):
    beams, vocab = 6, 9001
    x = _rand(5 * beams, vocab, dtype=dtype, seed=1, scale=3.0)
    x[torch.rand(x.shape, generator=torch.Generator().manual_seed(2)) < 0.5] = -math.inf
    scores = -10.0 * torch.rand(5 * beams, generator=torch.Generator().manual_seed(3))
    ended = torch.rand(5 * beams, generator=torch.Generator().manual_seed(4)) < 0.4
    ended[:beams] = True                                     # a group that has ended: fewer continuations than asked for
    x[beams:2 * beams] = -math.inf                           # a group without any
    ended[beams:2 * beams] = False
    scores[2 * beams + 1:3 * beams] = -math.inf              # the first step: one hypothesis lives
    ended[2 * beams:3 * beams] = False
    x[3 * beams, 5], x[3 * beams + 1, 7], scores[3 * beams + 2] = math.nan, math.inf, math.nan
    ended[3 * beams:] = False
    _select(x, scores, beams, 9, ended, end=17)


def test_select_ties_go_to_the_lowest():
    vocab = 20011
    for dtype in (F32, BF16):
        flat = torch.zeros(4, vocab, dtype=dtype)
        _select(flat, torch.tensor([0.0, 0.0, -1.0, 0.0]), 4, 13)
        few = torch.randint(0, 3, (4, vocab), generator=torch.Generator().manual_seed(1)).to(dtype)
        _select(few, torch.zeros(4), 2, 40)
        row = _rand(1, vocab, dtype=dtype, seed=5)           # hypotheses that are the same: odd rows start elsewhere in memory
        _select(row.repeat(8, 1), torch.full((8,), -3.7), 8, 20)
        zeros = torch.where(torch.arange(vocab) % 2 == 0, 0.0, -0.0).to(dtype).repeat(2, 1)
        _select(zeros, torch.zeros(2), 1, 11)


@pytest.mark.parametrize("dtype", [F32, F16])
def test_select_rows_that_rise_and_fall(dtype):
    """Orders that a running threshold meets at its worst: every element above all before it."""
    vocab = 30011
    up = torch.arange(vocab).float() / 4096
    x = torch.stack([up, up.flip(0), up, torch.full((vocab,), -3.0)]).to(dtype)
    _select(x, torch.tensor([0.0, -0.1, -0.25, 0.0]), 2, 31)


def test_select_views_large_offsets_and_streams():
    from paper_2402_09633_gb300 import beam_select
    wide = _rand(6, 5005, dtype=BF16, seed=3)
    dev = wide.cuda()
    scores = _rand(6, dtype=F32, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = beam_select(dev[:, 3:4004], scores.cuda(), 3, stream=side)
    side.synchronize()
    want = P.best(wide[:, 3:4004], scores, 3, 3)
    assert torch.equal(got[1].cpu().view(2, 3).long(), want[1]) and torch.equal(got[2].cpu().view(2, 3).long(), want[2])
    assert all(x.numel() == 0 for x in beam_select(dev[:0], scores[:0].cuda(), 3))


# ------------------------------------------------------------------------------------------- moving states

def _moved(x, parents, beams):
    at = torch.arange(x.shape[0]) // beams * beams + parents.long()
    return x[at]


@pytest.mark.parametrize("beams", [1, 2, 5, 16, 64])
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder_states(beams, in_place):
    from paper_2402_09633_gb300 import beam_reorder
    groups = 7
    n = groups * beams
    g = torch.Generator().manual_seed(beams)
    parents = torch.randint(0, beams, (n,), generator=g, dtype=torch.int32)
    parents[:beams] = torch.randperm(beams, generator=g).int()                   # a group that only changes places
    wide = _rand(n, 3, 50, dtype=BF16, seed=1)
    states = [_rand(n, 1000, dtype=F32, seed=2), torch.randint(0, 99, (n, 3, 7), generator=g, dtype=torch.int32), wide,
              torch.randint(0, 99, (n, 5), generator=g).to(torch.uint8), _rand(n, dtype=F32, seed=3), torch.zeros(n, 0),
              _rand(n, 70001, dtype=F16, seed=4)]
    dev = [x.cuda() for x in states]
    dev[2] = torch.zeros(n, 4, 50, dtype=BF16, device="cuda")[:, :3].copy_(wide) # rows apart
    out = None if in_place else [torch.empty_like(x) for x in dev]
    got = beam_reorder(parents.cuda(), beams, dev, out=out)
    for x, y, z in zip(got, states, dev):
        assert torch.equal(x.cpu(), _moved(y, parents, beams))
        assert in_place or torch.equal(z.cpu(), y)


def test_reorder_keeps_slots_whose_parent_is_none():
    from paper_2402_09633_gb300 import beam_reorder
    x = torch.arange(8.0).view(4, 2)
    got, = beam_reorder(_i32([1, -1, 2, 0]), 2, [x.cuda()])
    assert torch.equal(got.cpu(), x[[1, 1, 2, 2]])


@pytest.mark.parametrize("dtype,kv,dim", [(BF16, 2, 64), (F32, 1, 96), (F16, 3, 7)])
@pytest.mark.parametrize("page", [16, 128])
def test_reorder_caches(dtype, kv, dim, page):
    """Three layers: full pages are shared, begun ones copied, and every slot can go on by itself."""
    from paper_2402_09633_gb300 import PagedCache, beam_reorder
    beams, lengths = 6, [0, 5, page, page + 3, 3 * page + page // 2, 4 * page]
    n, width = beams * len(lengths), 5
    g = torch.Generator().manual_seed(page)
    parents = torch.randint(0, beams, (n,), generator=g, dtype=torch.int32)
    table, pages = _table(n, width, seed=1)
    pools = [tuple(_rand(pages * page, kv, dim, dtype=dtype, seed=10 * i + s) for s in (1, 2)) for i in range(3)]
    length = torch.tensor(lengths).repeat_interleave(beams).int()
    dev = [(k.cuda(), v.cuda()) for k, v in pools]
    on = table.cuda()
    caches = [PagedCache(k, v, on, length.cuda(), page) for k, v in dev]
    caches = [PagedCache(k, v, on, caches[0].kv_len, page) for k, v in dev]
    more = torch.arange(n).float()
    moved, = beam_reorder(parents.cuda(), beams, [more.cuda()], caches=caches)
    assert all(c.status() == 0 for c in caches) and torch.equal(moved.cpu(), _moved(more, parents, beams))
    new = on.cpu()
    for i in range(n):
        a, L = i - i % beams + int(parents[i]), int(length[i])
        full = L // page
        assert torch.equal(new[i, :full], table[a, :full]) and torch.equal(new[i, full:], table[i, full:])
        for (k, v), (k0, v0) in zip(dev, pools):
            for x, x0 in ((k, k0), (v, v0)):
                assert torch.equal(x.cpu()[P.rows_of(new, page, i, 0, L)], x0[P.rows_of(table, page, a, 0, L)])
    kept = torch.ones(pages * page, dtype=torch.bool)        # nothing else is written
    for i in range(n):
        full = int(length[i]) // page
        if int(length[i]) % page:
            kept[int(table[i, full]) * page:int(table[i, full]) * page + int(length[i]) % page] = False
    for (k, v), (k0, v0) in zip(dev, pools):
        assert torch.equal(k.cpu()[kept], k0[kept]) and torch.equal(v.cpu()[kept], v0[kept])


def test_reorder_reports_groups_that_cannot_be_moved():
    from paper_2402_09633_gb300 import PagedCache, beam_reorder, binding
    page = 16
    k = _rand(8 * page, 1, 32, dtype=F32, seed=1)
    for table, length, parents in (([[0, 1], [2, 3]], [17, 18], [1, 0]), ([[0, 9], [2, 3]], [17, 17], [1, 0]),
                                   ([[0, 1], [2, 3]], [33, 33], [1, 1]), ([[0, 1], [2, 3]], [-1, -1], [1, 1]),
                                   ([[0, 1], [2, 3]], [17, 17], [2, 1])):
        on, dk, dv = torch.tensor(table, dtype=torch.int32).cuda(), k.cuda(), k.cuda()
        cache = PagedCache(dk, dv, on, _i32(length), page)
        beam_reorder(_i32(parents), 2, caches=[cache])
        assert binding.ERRORS[cache.status()] == "INDEX_RANGE"
        assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), k) and on.cpu().tolist() == table


# ------------------------------------------------------------------------------------------- together

def _steps(graph):
    """Beam search over two layers of caches, against the same search with whole sequences of keys kept apart."""
    from paper_2402_09633_gb300 import PagedCache, Rotary, beam_reorder, beam_select
    E, B, V, H, K, D, page, S, steps = 3, 4, 50, 4, 2, 64, 16, [40, 33, 64], 20
    n = E * B
    g = torch.Generator().manual_seed(0)
    dt = BF16
    width = 8
    table, pages = _table(n, width, seed=1)
    for e in range(E):                                       # whole pages of an event's tokens are one for all its hypotheses
        table[e * B:(e + 1) * B, :S[e] // page] = table[e * B, :S[e] // page]
    emb = _rand(V, 3 * 64, dtype=dt, seed=2)                 # of a token: what its q, k, v come from
    weights = [(_rand(64, (H + 2 * K) * D, dtype=dt, seed=3 + i, scale=0.2), _rand(H * D, V, dtype=dt, seed=7 + i, scale=0.3)) for i in range(2)]
    kc = [(torch.zeros(pages * page, K, D, dtype=dt, device="cuda"), torch.zeros(pages * page, K, D, dtype=dt, device="cuda")) for _ in range(2)]
    on, length = table.cuda(), _i32([0] * n)
    caches = [PagedCache(k, v, on, length, page) for k, v in kc]
    rot, table_of = Rotary(D), emb.cuda()
    cw = [(a.cuda(), b.cuda()) for a, b in weights]
    prompt = torch.randint(0, V, (E, max(S)), generator=g)

    def project(tokens, i):
        x = table_of[tokens][:, 64 * i:64 * i + 64] @ cw[i][0]
        x = x.view(-1, H + 2 * K, D)
        return x[:, :H], x[:, H:H + K], x[:, H + K:]

    # the events' tokens, by the first hypothesis; the last page's rows by all
    for e in range(E):
        for b in range(B):
            length.zero_()
            length[e * B + b] = S[e]
            start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
            start[e * B + b + 1:] = S[e]
            toks = prompt[e, :S[e]].cuda()
            for i in range(2):
                _, k, v = project(toks, i)
                caches[i].append(rot, start, k.contiguous(), v.contiguous())
    length.copy_(_i32([S[i // B] for i in range(n)]))
    groups, shared = _i32([0, B, 2 * B, 3 * B]), _i32(S)
    each = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    token = _i32([int(prompt[i // B, S[i // B] - 1]) for i in range(n)])
    scores = torch.tensor([0.0 if i % B == 0 else -math.inf for i in range(n)], device="cuda")
    history = torch.full((n, steps), -1, dtype=torch.int32, device="cuda")
    at = torch.zeros(1, dtype=torch.long, device="cuda")

    def step():
        length.add_(1)
        x = None
        for i in range(2):
            q, k, v = project(token.long(), i)
            q = caches[i].append(rot, each, k, v, q=q, eps=1e-6)
            o = caches[i].attend(q, each, groups=groups, shared=shared, max_q=1)
            y = o.reshape(n, H * D) @ cw[i][1]
            x = y if x is None else x + y
        s, p, t = beam_select(x, scores, B)
        beam_reorder(p, B, [history], caches=caches)
        history.index_copy_(1, at, t[:, None])
        scores.copy_(s)
        token.copy_(t)
        at.add_(1)
        return x, p

    # plain: every hypothesis' tokens kept whole
    def plain(tokens_of):
        out = torch.zeros(n, V, dtype=torch.float64)
        for r in range(n):
            toks = torch.tensor(tokens_of[r])
            for i in range(2):
                q, k, v = (x.double().cpu() for x in project(toks.cuda(), i))
                pos = torch.arange(len(toks))
                first = S[r // B]
                kk = k.clone()
                kk[first:] = R.norm(k[first:], None, 1e-6)
                kk, _ = R.rotate(kk, pos, D, "half")
                qq, _ = R.rotate(R.norm(q[-1:], None, 1e-6), pos[-1:], D, "half")
                w = torch.softmax((qq.transpose(0, 1) @ kk.permute(1, 2, 0).repeat_interleave(H // K, 0)) / math.sqrt(D), -1)
                o = (w @ v.permute(1, 0, 2).repeat_interleave(H // K, 0)).transpose(0, 1).reshape(1, H * D)
                out[r] += (o @ weights[i][1].double())[0]
        return out

    seqs = [prompt[r // B, :S[r // B]].tolist() for r in range(n)]
    last = [s[-1] for s in seqs]
    run = step
    captured = None
    for it in range(steps):
        if graph and it == 1:
            keep = [x.clone() for x in (length, token, scores, history, at, on, *kc[0], *kc[1])]
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                res = step()
            for x, y in zip((length, token, scores, history, at, on, *kc[0], *kc[1]), keep):
                x.copy_(y)
        seqs = [s + [t] for s, t in zip(seqs, last)]
        before = scores.cpu()
        if captured is not None:
            captured.replay()
            x, p = res
        else:
            x, p = run()
        want = plain(seqs)
        live = before > -math.inf
        got = x.double().cpu()
        # roundings to bf16 at each product, norm, weight and output
        assert float((got - want)[live].abs().max()) <= 16 * 2.0 ** -8 * float(want[live].abs().max())
        pick = P.best(x.cpu(), before, B, B)
        assert torch.equal(p.cpu().view(E, B).long(), pick[1]) and torch.equal(token.cpu().view(E, B).long(), pick[2])
        par, tok = p.cpu().tolist(), token.cpu().tolist()
        seqs = [list(seqs[r // B * B + par[r]]) for r in range(n)]
        last = tok
    assert all(c.status() == 0 for c in caches)
    for r in range(n):
        assert history[r].cpu().tolist() == seqs[r][S[r // B] + 1:] + [last[r]]


@pytest.mark.parametrize("graph", [False, True])
def test_beam_search_steps(graph):
    _steps(graph)
