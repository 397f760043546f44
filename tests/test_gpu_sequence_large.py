"""Sequence operators where counts and offsets are large: many sequences, many blocks of work to an SM, and views
whose rows lie more than 2^32 bytes apart."""
import math

import pytest
import torch

from tests import sequence_ref as R
from tests.test_gpu_sequence import _attend, _rand, _starts

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("seqs,H,K,D,nq,most,left", [
    (129, 4, 2, 64, 1, 90, -1), (700, 2, 1, 32, 2, 40, 9), (1024, 3, 1, 64, 1, 130, 70), (1025, 8, 8, 64, 1, 33, -1),
    (3000, 16, 2, 16, 3, 20, 5), (90, 8, 1, 128, 1, 5000, -1), (3, 40, 2, 96, 1, 9000, -1)])
def test_many_sequences_over_caches(seqs, H, K, D, nq, most, left):
    g = torch.Generator().manual_seed(seqs)
    nk = torch.randint(0, most, (seqs,), generator=g).tolist()
    q = _rand(seqs * nq, H, D, dtype=BF16, seed=1)
    k, v = (_rand(sum(nk) + 1, K, D, dtype=BF16, seed=s) for s in (2, 3))
    _attend(q, k, v, _starts([nq] * seqs), _starts(nk)[:-1], nk, left, 0, 2, max_q=nq)


@pytest.mark.parametrize("H,K,D", [(3, 3, 64), (4, 2, 128)])
def test_many_tiles_to_a_block(H, K, D):
    lengths = [int(x) for x in torch.randint(0, 900, (60,), generator=torch.Generator().manual_seed(4))]
    q, k, v = (_rand(sum(lengths), h, D, dtype=F16, seed=h + 1) for h in (H, K, K))
    _attend(q, k, v, _starts(lengths), None, None, 60, 33, 3)


@pytest.mark.parametrize("max_q", [1, 0])
def test_offsets_beyond_32_bits(max_q):
    rows, step = 700, 5_000_000                              # 7 GB from the first row to the last
    area = torch.empty(2, rows * step, dtype=BF16, device="cuda")
    k, v = (_rand(rows, 1, 64, dtype=BF16, seed=s) for s in (1, 2))
    far = [a.as_strided((rows, 1, 64), (step, 64, 1)) for a in area]
    for x, y in zip(far, (k, v)):
        x.copy_(y.cuda())
    n = 1 if max_q else 130
    q = _rand(n, 1, 64, dtype=BF16, seed=3)
    got = _attend(q, k, v, [0, n], [0], [rows], -1, 0, 0, dev=(q.cuda(), *far), max_q=max_q)
    assert torch.isfinite(got).all()
    from paper_2402_09633_gb300 import Rotary, qk_norm_rope, rope
    pos = torch.arange(rows)
    want = R.rotate(k, pos, 64, "half")
    rope(Rotary(64), far[0], out=far[0])
    R.check_rotated(far[0].cpu(), *want, normed=False)
    slots = torch.arange(rows, device="cuda").flip(0)
    qkv = _rand(rows, 3, 64, dtype=BF16, seed=4)
    dev = qkv.cuda()
    qk_norm_rope(Rotary(64), dev[:, :1], dev[:, 1:2], v=dev[:, 2:], k_out=far[0], v_out=far[1], rows=slots)
    R.check_rotated(far[0].cpu().flip(0), *R.rotate(R.norm(qkv[:, 1:2], None, 1e-6), pos, 64, "half"), normed=True)
    assert torch.equal(far[1].cpu().flip(0), qkv[:, 2:])


def test_a_row_that_is_not_finite_costs_only_itself():
    """An event with values that are not finite beside others in one batch: the others' results do not change."""
    lengths = [333, 500, 290]
    q, k, v = (_rand(sum(lengths), 2, 64, dtype=BF16, seed=s) for s in (1, 2, 3))
    clean = _attend(q, k, v, _starts(lengths), None, None, 100, 100, 4)
    v2, k2 = v.clone(), k.clone()
    v2[333:833] = math.nan
    k2[333:833] = math.inf
    got = _attend(q, k2, v2, _starts(lengths), None, None, 100, 100, 4)
    assert torch.equal(got[:333], clean[:333]) and torch.equal(got[833:], clean[833:])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("H,K,nq", [(4, 1, 4), (2, 2, 3), (16, 2, 5)])
def test_new_queries_that_see_different_keys(dtype, H, K, nq):
    """Several new queries of a sequence: a key that one of them sees may hold anything for the others."""
    n = 777
    q, k, v = (_rand(r, h, 64, dtype=dtype, seed=h + r) for r, h in ((nq, H), (n, K), (n, K)))
    v[n - 1, 0, 5] = math.nan                                # the last query's own key
    v[n - 2, 0] = math.inf                                   # seen by the last two
    k[n - nq - 50] = math.nan                                # at the left edge of the first
    _attend(q, k, v, [0, nq], [0], [n], 50, 0, 0, max_q=nq, max_kv=n)
    _attend(q, k, v, [0, nq], [0], [n], 50, 0, 3, max_q=nq, max_kv=n)


@pytest.mark.parametrize("rows,most", [(300, 100), (2, 1)])
def test_more_queries_than_announced_are_reported(rows, most):
    from paper_2402_09633_gb300 import WindowAttention
    x = torch.zeros(rows, 1, 64, dtype=BF16, device="cuda")
    att, starts = WindowAttention(), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    att(x, x, x, starts, left=10, right=0, max_q=most)
    assert att.status() == -5
    att(x, x, x, starts, left=10, right=0, max_q=rows)
    assert att.status() == 0
