"""Rotary positions, norms of queries and keys with the rotation, and attention with a sliding window on the GPU
against plain statements in 64 bits, at the sizes, layouts and masks where they can go wrong."""
import math

import pytest
import torch

from tests import sequence_ref as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _rand(*size, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*size, generator=g) * scale).to(dtype)


# ------------------------------------------------------------------------------------------- rope

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,dim,rot", [
    (1, 1, 2, 2), (3, 2, 64, 64), (257, 3, 64, 20), (130, 2, 96, 40), (33, 5, 128, 128), (65, 1, 128, 30),
    (9, 2, 256, 256), (17, 1, 250, 2), (40, 7, 64, 62), (5000, 2, 32, 16)])
def test_rope(dtype, layout, rows, heads, dim, rot):
    from paper_2402_09633_gb300 import Rotary, rope
    x = _rand(rows, heads, dim, dtype=dtype, seed=rows + dim)
    pos = torch.randint(-5, 300000, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    got = rope(Rotary(rot, layout=layout), x.cuda(), pos.cuda())
    R.check_rotated(got, *R.rotate(x, pos, rot, layout), normed=False)


@pytest.mark.parametrize("scaling", [None, ("linear", 4.0), ("turns", 8.0, 32768.0, 1.0, 32.0)])
@pytest.mark.parametrize("base,amplitude", [(10000.0, 1.0), (500000.0, 1.25)])
def test_rope_scalings_and_extreme_positions(scaling, base, amplitude):
    from paper_2402_09633_gb300 import Rotary, rope
    pos = torch.tensor([0, 1, -1, 4095, 4096, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32)
    x = _rand(pos.numel(), 2, 128, dtype=F32, seed=4)
    got = rope(Rotary(128, base, "half", scaling, amplitude), x.cuda(), pos.cuda())
    R.check_rotated(got, *R.rotate(x, pos, 128, "half", base, scaling, amplitude), normed=False)


def test_rope_real_positions_row_numbers_views_and_in_place():
    from paper_2402_09633_gb300 import Rotary, rope
    rot = Rotary(32, layout="interleaved")
    pos = _rand(100, dtype=F32, seed=1, scale=50.0)
    wide = _rand(100, 9, 64, dtype=BF16, seed=2)
    x = wide[:, 3:6, :48]                                    # a slice: row and head strides of its own
    dev = wide.cuda()
    want = R.rotate(x, pos, 32, "interleaved")
    R.check_rotated(rope(rot, dev[:, 3:6, :48], pos.cuda()), *want, normed=False)
    rope(rot, dev[:, 3:6, :48], pos.cuda(), out=dev[:, 3:6, :48])
    R.check_rotated(dev[:, 3:6, :48].cpu(), *want, normed=False)
    untouched = torch.ones(100, 9, 64, dtype=torch.bool)
    untouched[:, 3:6, :48] = False
    assert torch.equal(dev.cpu()[untouched], wide[untouched])
    odd = _rand(100 * 3 * 50 + 1, dtype=BF16, seed=3)[1:].view(100, 3, 50)     # 2-byte aligned
    on_gpu = torch.empty(100 * 3 * 50 + 1, dtype=BF16, device="cuda")[1:].view(100, 3, 50)
    on_gpu.copy_(odd)
    R.check_rotated(rope(rot, on_gpu), *R.rotate(odd, torch.arange(100), 32, "interleaved"), normed=False)
    heads_first = _rand(4, 77, 64, dtype=F16, seed=5)
    R.check_rotated(rope(Rotary(64), heads_first.cuda().transpose(0, 1)),
                    *R.rotate(heads_first.transpose(0, 1), torch.arange(77), 64, "half"), normed=False)
    empty = torch.empty(0, 3, 64, device="cuda")
    assert rope(rot, empty).shape == (0, 3, 64)


# ------------------------------------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,kv,dim,rot,gains", [
    (1, 1, 1, 2, 2, True), (64, 16, 4, 128, 128, True), (1000, 6, 2, 96, 40, True), (77, 3, 1, 250, 30, False),
    (4099, 2, 2, 64, 64, True), (5, 8, 8, 256, 256, True), (31, 1, 1, 6, 4, False)])
def test_qk_norm_rope(dtype, layout, rows, heads, kv, dim, rot, gains):
    from paper_2402_09633_gb300 import Rotary, qk_norm_rope
    qkv = _rand(rows, heads + 2 * kv, dim, dtype=dtype, seed=rows, scale=3.0)
    qkv[0, 0] = 0                                            # a head of zeros stays zero
    pos = torch.randint(0, 100000, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    gq, gk = (1 + _rand(dim, dtype=F32, seed=s, scale=0.3) for s in (1, 2)) if gains else (None, None)
    cu = lambda x: None if x is None else x.cuda()           # noqa: E731
    dev = qkv.cuda()
    got = qk_norm_rope(Rotary(rot, layout=layout), dev[:, :heads], dev[:, heads:heads + kv], pos.cuda(),
                       v=dev[:, heads + kv:], q_gain=cu(gq), k_gain=cu(gk), eps=1e-5)
    for g, x, gain in ((got[0], qkv[:, :heads], gq), (got[1], qkv[:, heads:heads + kv], gk)):
        R.check_rotated(g, *R.rotate(R.norm(x, gain, 1e-5), pos, rot, layout), normed=True)
    assert torch.equal(got[2].cpu(), qkv[:, heads + kv:])


def test_norm_places_keys_and_values_in_cache_rows():
    from paper_2402_09633_gb300 import Rotary, qk_norm_rope
    n, kv, dim, cap = 300, 2, 64, 1000
    q, k, v = (_rand(n, h, dim, dtype=BF16, seed=h + 3) for h in (4, kv, kv))
    rows = torch.randperm(cap, generator=torch.Generator().manual_seed(0))[:n]
    rows[7], rows[8] = -1, cap                               # not written
    kc, vc = (_rand(cap, kv, dim, dtype=BF16, seed=s) for s in (8, 9))
    gk, gv = kc.cuda(), vc.cuda()
    qkv = [x.cuda() for x in (q, k, v)]
    out = qk_norm_rope(Rotary(64), qkv[0], qkv[1], v=qkv[2], k_out=gk, v_out=gv, rows=rows.cuda())
    assert out[1].data_ptr() == gk.data_ptr() and out[2].data_ptr() == gv.data_ptr()
    pos = torch.arange(n)
    want, size = R.rotate(R.norm(k, None, 1e-6), pos, 64, "half")
    live = (rows >= 0) & (rows < cap)
    R.check_rotated(gk.cpu()[rows[live]], want[live], size[live], normed=True)
    assert torch.equal(gv.cpu()[rows[live]], v[live])
    rest = torch.ones(cap, dtype=torch.bool)
    rest[rows[live]] = False
    assert torch.equal(gk.cpu()[rest], kc[rest]) and torch.equal(gv.cpu()[rest], vc[rest])
    R.check_rotated(out[0], *R.rotate(R.norm(q, None, 1e-6), pos, 64, "half"), normed=True)
    # without values, in place
    qk_norm_rope(Rotary(64), qkv[0], qkv[1], q_out=qkv[0], k_out=qkv[1])
    R.check_rotated(qkv[1], want, size, normed=True)


# ------------------------------------------------------------------------------------------- attention

def _attend(q, k, v, q_start, kv_start, kv_len, left, right, sinks, scale=None, dev=None, **kw):
    from paper_2402_09633_gb300 import WindowAttention
    att = WindowAttention()
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    dq, dk, dv = dev or (x.cuda() for x in (q, k, v))
    own = kv_start is None
    got = att(dq, dk, dv, i32(q_start), left=left, right=right, sinks=sinks, scale=scale, kv_start=i32(kv_start),
              kv_len=i32(kv_len), **kw).cpu()
    assert att.status() == 0
    att.close()
    if own:
        kv_start, kv_len = q_start[:-1], [z - a for a, z in zip(q_start, q_start[1:])]
    R.check_attention(got, q, k, v, q_start, kv_start, kv_len, left, right, sinks,
                      1 / math.sqrt(q.shape[2]) if scale is None else scale)
    return got


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return s


PACKED = [  # lengths, heads, kv heads, dim, left, right, sinks
    ([1], 1, 1, 64, -1, -1, 0),
    ([1], 2, 1, 128, 0, 0, 0),
    ([127], 2, 2, 64, -1, -1, 0),
    ([128], 2, 2, 64, -1, 0, 0),
    ([129], 1, 1, 64, 0, 0, 0),
    ([300], 2, 2, 64, 16, 16, 4),
    ([300], 4, 2, 128, 31, 0, 3),
    ([257, 0, 1, 130, 64], 3, 1, 64, 100, 50, 2),
    ([257, 0, 1, 130, 64], 6, 2, 96, 100, 0, 200),
    ([700], 8, 1, 128, 127, 0, 129),
    ([700], 2, 1, 40, 128, 128, 1),
    ([515], 1, 1, 8, 3, 250, 40),
    ([640], 2, 2, 72, 300, -1, 7),
    ([640], 5, 5, 64, -1, 130, 0),
    ([1100], 2, 1, 64, 200, 700, 5),
    ([1100], 3, 3, 128, 1000, 0, 16),
    ([5, 3, 9, 2, 11, 1, 0, 0, 4] * 6, 4, 4, 64, 2, 2, 1),
    ([900, 33], 16, 2, 16, 64, 64, 64),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("case", range(len(PACKED)))
def test_packed_sequences(case, dtype):
    lengths, H, K, D, left, right, sinks = PACKED[case]
    n = sum(lengths)
    qkv = _rand(n, H + 2 * K, D, dtype=dtype, seed=case)
    dev = qkv.cuda()                                         # slices of a packed projection
    cut = lambda x: (x[:, :H], x[:, H:H + K], x[:, H + K:])  # noqa: E731
    _attend(*cut(qkv), _starts(lengths), None, None, left, right, sinks, dev=cut(dev))


CACHED = [  # queries, keys, capacity, heads, kv heads, dim, left, right, sinks
    ([1], [1], 1, 1, 1, 64, -1, 0, 0),
    ([1], [4097], 4099, 4, 1, 128, 1023, 0, 4),
    ([1, 1, 1], [0, 5, 300], 300, 16, 4, 128, -1, 0, 0),
    ([3, 3], [2, 700], 701, 8, 2, 64, -1, 0, 0),                    # more queries than keys: the first sees none
    ([1, 2, 0, 4], [100, 1000, 50, 3], 1000, 6, 2, 96, 40, 0, 7),
    ([1] * 9, [17, 333, 1024, 1, 2, 900, 31, 32, 33], 1024, 12, 3, 40, 64, 0, 64),
    ([7], [2000], 2000, 2, 2, 64, -1, -1, 0),
    ([1], [70001], 70001, 8, 8, 8, -1, 0, 0),
    ([2, 2], [9000, 8000], 9000, 32, 2, 128, -1, 0, 0),
    ([200, 1], [300, 600], 600, 4, 2, 64, 128, 0, 16),              # a chunk of a prompt beside a step
    ([5, 5], [400, 10], 400, 2, 1, 64, 3, 2, 1),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("known", [False, True])
@pytest.mark.parametrize("case", range(len(CACHED)))
def test_queries_over_a_cache(case, known, dtype):
    nq, nk, cap, H, K, D, left, right, sinks = CACHED[case]
    q = _rand(sum(nq), H, D, dtype=dtype, seed=case)
    k, v = (_rand(len(nq) * cap, K, D, dtype=dtype, seed=s + case) for s in (50, 90))
    starts = [b * cap for b in range(len(nq))]
    for b, n in enumerate(nk):                               # what lies behind a sequence's last key counts for nothing
        k[starts[b] + n:starts[b] + cap] = math.nan
        v[starts[b] + n:starts[b] + cap] = math.nan
    bounds = {"max_q": max(nq), "max_kv": max(nk)} if known else {}
    _attend(q, k, v, _starts(nq), starts, nk, left, right, sinks, **bounds)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("cached", [False, True])
def test_not_finite_values_reach_only_queries_that_see_them(cached, dtype):
    H, K, D = 2, 1, 64
    lengths = [300, 200]
    q, k, v = (_rand(500, h, D, dtype=dtype, seed=h + 20) for h in (H, K, K))
    v[40, 0, 3] = math.nan
    v[77, 0, 9] = math.inf
    v[310, 0] = -math.inf
    k[450, 0, 5] = math.nan
    k[120] = math.nan
    q[200, 1, 0] = math.nan
    if cached:
        pick = [60, 150, 299]
        for p in pick:                                       # a single query at each place, its keys before it
            _attend(q[p:p + 1], k, v, [0, 1], [0], [p + 1], 30, 0, 2)
        return
    got = _attend(q, k, v, _starts(lengths), None, None, 10, 10, 2)
    assert torch.isfinite(got[100]).all() and torch.isfinite(got[299]).all()


@pytest.mark.parametrize("cached", [False, True])
def test_large_scores_and_scales(cached):
    n, H, K, D = 260, 2, 2, 64
    for scale, size in ((1.0, 6.0), (0.0, 1.0), (-0.3, 2.0)):
        q, k, v = (_rand(n, h, D, dtype=BF16, seed=h + 31, scale=size) for h in (H, K + 0, K))
        if cached:
            _attend(q[-1:], k, v, [0, 1], [0], [n], -1, 0, 0, scale=scale)
        else:
            _attend(q, k, v, [0, n], None, None, 100, 0, 5, scale=scale)


def test_growing_scores_rescale_the_sums():
    """Keys whose scores grow along the sequence: every block raises the running maximum."""
    n, D = 1500, 64
    q = torch.ones(n, 1, D, dtype=BF16)
    k = (torch.arange(n, dtype=torch.float32)[:, None, None] / 16).expand(n, 1, D).to(BF16).contiguous()
    v = _rand(n, 1, D, dtype=BF16, seed=1)
    _attend(q, k, v, [0, n], None, None, -1, 0, 0, scale=1 / 16)
    _attend(q, k.flip(0).contiguous(), v, [0, n], None, None, -1, -1, 0, scale=1 / 16)
    _attend(q[-2:], k, v, [0, 2], [0], [n], -1, 0, 0, scale=1 / 16)


def test_strided_views_of_either_order():
    H, K, D, n = 4, 2, 64, 333
    q, k, v = (_rand(h, n, D, dtype=BF16, seed=h).transpose(0, 1) for h in (H, K, K))   # heads before rows
    dev = [x.transpose(0, 1).cuda().transpose(0, 1) for x in (q, k, v)]
    wide = torch.zeros(n, H + 3, D + 8, dtype=BF16, device="cuda")
    out = wide[:, 1:1 + H, :D]
    got = _attend(q, k, v, [0, n], None, None, 50, 20, 3, dev=dev, out=out)
    assert torch.equal(wide[:, 1:1 + H, :D].cpu(), got)
    wide[:, 1:1 + H, :D] = 0
    assert not wide.any()


def test_rows_outside_the_sequences_are_not_written():
    q, k, v = (_rand(400, 2, 64, dtype=F16, seed=s) for s in (1, 2, 3))
    from paper_2402_09633_gb300 import WindowAttention
    att = WindowAttention()
    out = torch.full((400, 2, 64), 7.0, dtype=F16, device="cuda")
    att(q.cuda(), k.cuda(), v.cuda(), torch.tensor([50, 50, 210], dtype=torch.int32, device="cuda"), left=20, right=5,
        out=out)
    assert att.status() == 0
    got = out.cpu()
    assert bool((got[:50] == 7).all()) and bool((got[210:] == 7).all())
    R.check_attention(got, q, k, v, [50, 210], [50], [160], 20, 5, 0, 0.125)


@pytest.mark.parametrize("max_q", [0, 1])
def test_offsets_outside_the_views_are_reported(max_q):
    from paper_2402_09633_gb300 import WindowAttention
    att = WindowAttention()
    x = torch.zeros(20, 1, 64, dtype=BF16, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")     # noqa: E731
    out = torch.zeros_like(x)
    for start, ks, kl in (([0, 1], [-4], [9]), ([0, 1], [0], [21]), ([0, 1], [19], [2]), ([0, 1], [0], [-3]),
                          ([0, 1], [2 ** 31 - 1], [2 ** 31 - 1])):
        att(x, x, x, i32(start), kv_start=i32(ks), kv_len=i32(kl), max_q=max_q, out=out)
        assert att.status() == -5
    att(x, x, x, i32([0, 1]), kv_start=i32([0]), kv_len=i32([20]), max_q=max_q, out=out)
    assert att.status() == 0


def test_runs_repeat_bit_for_bit_on_any_stream_and_in_a_graph():
    from paper_2402_09633_gb300 import WindowAttention
    q, k, v = (_rand(3000, h, 128, dtype=BF16, seed=h).cuda() for h in (8, 2, 2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
    att = WindowAttention()
    calls = [dict(q=q, q_start=i32([0, 1000, 3000]), left=200, right=0, sinks=4),
             dict(q=q[:2], q_start=i32([0, 1, 2]), kv_start=i32([0, 900]), kv_len=i32([800, 2100]), max_q=1)]
    for c in calls:
        first = att(k=k, v=v, **c)
        again = att(k=k, v=v, **c)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            there = WindowAttention()(k=k, v=v, **c)
        side.synchronize()
        out = torch.empty_like(first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            att(k=k, v=v, out=out, **c)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, again) and torch.equal(first, there) and torch.equal(first, out)
    assert att.status() == 0


def test_no_queries_no_sequences_no_keys():
    from paper_2402_09633_gb300 import WindowAttention
    att = WindowAttention()
    e = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    q = torch.ones(3, 2, 64, dtype=BF16, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
    assert att(e, e, e, i32([0])).shape == (0, 2, 64)
    assert att(e, e, e, i32([0, 0])).shape == (0, 2, 64)
    got = att(q, e, e, i32([0, 3]), kv_start=i32([0]), kv_len=i32([0]))
    assert att.status() == 0 and not got.any()
    got = att(q, e, e, i32([0, 1, 3]), kv_start=i32([0, 0]), kv_len=i32([0, 0]), max_q=2)
    assert att.status() == 0 and not got.any()
