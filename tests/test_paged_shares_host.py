"""How the attention over pages shares out its blocks of keys (csrc/paged_tile.cuh), run on the CPU from its own source: every
block of every item is taken once, shares are even, and what the parts leave lies apart and inside the workspace."""
import ctypes

import numpy as np
import pytest

from tests import host_cuda

MAIN = r"""
#include "ptx.cuh"
#include <climits>
#include <cmath>
using std::max;
using std::min;
struct int2 { int x, y; };
inline int2 make_int2(int x, int y) { return {x, y}; }
inline int64_t __shfl_up_sync(unsigned m, int64_t x, int by) {
  const uint32_t lo = __shfl_up_sync(m, (uint32_t)x, by), hi = __shfl_up_sync(m, (uint32_t)(x >> 32), by);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
#define __grid_constant__
namespace gnn { inline void pdl_trigger() {} }
#include "shares.cuh"
using namespace gnn;
// out: own, index, item, b0, b1, first thread block, parts, ordinal, thread block, blocks, both
extern "C" int walk(int grid, int n_q, int n_seqs, int n_groups, const int* q_start, const int* kv_len, const int* group_start,
                    const int* shared, int max_q, int kv_heads, int group, int pack, int page, int width, long long* out, int most, unsigned* err,
                    long long* share_out, int counted) {
  PagedParams p = {};
  p.q_start = q_start; p.kv_len = kv_len; p.group_start = group_start; p.shared_len = shared;
  p.n_q_rows = n_q; p.n_seqs = n_seqs; p.n_groups = n_groups; p.width = width; p.max_q = max_q;
  p.kv_heads = kv_heads; p.heads = kv_heads * group; p.err = err;
  while (1 << p.shift < page) ++p.shift;
  PagedGrid g = {};
  g.group = group; g.tile_q = kTileQ / group; g.box = min(page, kKeys); g.pack = pack;
  const int n_chunks = (n_seqs + kAttendThreads - 1) / kAttendThreads + (n_groups + kAttendThreads - 1) / kAttendThreads;
  std::vector<int64_t> chunks(n_chunks, -1);
  if (n_seqs > kPagedKept || n_groups > kAttendThreads || counted) g.chunks = chunks.data();
  static PagedBars bars;
  int n = 0;
  gridDim.x = n_chunks;
  if (g.chunks) host::launch(n_chunks, kAttendThreads, [&] { paged_weigh_kernel(p, g); });
  gridDim.x = grid;
  host::launch(grid, kAttendThreads, [&] {
    if (threadIdx.x == 0) { bars.at = -1000000; bars.before = -7; }           // shared memory holds anything at first
    __syncthreads();
    const PagedShare share = paged_share(p, g, bars);
    if (share.start >= share.end && share.before < share.end) std::abort();
    if (threadIdx.x == 0) *share_out = share.share;
    if (threadIdx.x >= 32) return;
    bool ok = true;
    auto part = [&](const PagedWork& w, bool own, int index, uint32_t s, int b0, int b1, int64_t u0, const PagedOwn& mine,
                    int prefix) {
      if (threadIdx.x != 0 || n >= most) return;
      const uint32_t e = s / kv_heads;
      const int both = e < (uint32_t)w.twos;
      const int64_t last = u0 + w.blocks - 1;
      const int64_t ordinal = ((own ? paged_ordinal_b(g, index, w.q0) : paged_ordinal_a(g, index, w.q0)) + e) * kv_heads + s % kv_heads;
      const long long row[11] = {own, index, s, b0, b1, (long long)blockIdx.x, (last - share.start) / share.share + 1, ordinal,
                                 (long long)blockIdx.x, w.blocks, both};
      for (int i = 0; i < 11; ++i) out[(long long)n * 11 + i] = row[i];
      ++n;
    };
    paged_walk(p, g, share, bars, part, ok);
  });
  return n;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cut = host_cuda.between
    rotary, tile = host_cuda.source("rotary.cuh"), host_cuda.source("paged_tile.cuh")
    text = "namespace gnn {\n"
    text += cut(rotary, "struct HeadsView {", "struct PagedPlace {")
    text += "constexpr int kTileQ = 128, kKeys = 128, kAttendThreads = 384;\n"
    text += cut(host_cuda.source("paged.cuh"), "struct PagedParams {", "// The row of position j")
    text += cut(tile, "constexpr int kPagedCost", "// A part of an item, as")
    text += "struct PagedBars { int64_t scan[2][12]; int64_t before; int at; PagedOwn own[kPagedKept]; PagedWork shared[kGroupsKept]; };\n"
    text += cut(tile, "// Block b's share of the list", "template <typename T, int DP>\n__global__")
    lib = host_cuda.compile_host(tmp_path_factory.mktemp("host"), MAIN, [("shares.cuh", text + "}\n")])
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.walk.argtypes = [i] * 4 + [vp] * 4 + [i] * 6 + [vp, i, vp, vp, i]
    lib.walk.restype = i
    return lib


def _pack(max_q, group):
    n = 1
    while n < 32 and 2 * n * max_q <= 128 // group:
        n *= 2
    return n


def _walk(lib, grid, nq, kv_len, groups, shared, kv_heads, group, page, max_q=None, width=None, n_q=None, q_start=None, counted=0):
    i32 = lambda x: np.ascontiguousarray(x, dtype=np.int32)  # noqa: E731
    q_start = i32(np.concatenate([[0], np.cumsum(nq)])) if q_start is None else i32(q_start)
    kv_len, groups, shared = i32(kv_len), i32(groups), i32(shared)
    n_q = int(q_start[-1]) if n_q is None else n_q
    width = -(-int(kv_len.max()) // page) if width is None else width
    out, err, share = np.zeros((400000, 11), np.int64), np.zeros(1, np.uint32), np.zeros(1, np.int64)
    at = lambda a: a.ctypes.data_as(ctypes.c_void_p)         # noqa: E731
    n = lib.walk(grid, n_q, kv_len.size, shared.size, at(q_start), at(kv_len), at(groups), at(shared),
                 int(max(nq)) if max_q is None else max_q, kv_heads, group,
                 _pack(int(max(nq)) if max_q is None else max_q, group), page, width, at(out), len(out), at(err), at(share), counted)
    return out[:n], int(err[0]), int(share[0]), n_q


def _bounds(n_q, n_seqs, n_groups, kv_heads, group, pack):
    tile_q = 128 // group
    return {0: (n_q // (2 * tile_q) + n_groups) * kv_heads,
            1: (-(-n_seqs // pack) if pack > 1 else n_q // tile_q + n_seqs) * kv_heads}


def _check(out, share, grid, bound):
    items, places, load = {}, set(), np.zeros(grid, np.int64)
    for own, index, s, b0, b1, first, parts, ordinal, block, blocks, both in out.tolist():
        assert 0 <= ordinal < bound[own] and (own, ordinal + block) not in places
        places.add((own, ordinal + block))                   # so places are below the bound and the grid
        items.setdefault((own, index, s), []).append((b0, b1, first, parts, ordinal, block, blocks))
        load[block] += b1 - b0
    assert load.max(initial=0) <= share
    for key, parts in items.items():
        parts.sort()
        assert parts[0][0] == 0 and parts[-1][1] == parts[0][6]
        assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
        assert [p[5] for p in parts] == list(range(parts[0][2], parts[0][2] + parts[0][3]))     # where the join looks for them
        assert len({p[4] for p in parts}) == 1
    return items


@pytest.mark.parametrize("grid", [1, 7, 152])
@pytest.mark.parametrize("seed", range(12))
def test_every_block_once(lib, grid, seed):
    rng = np.random.default_rng(seed)
    n = int([1, 3, 31, 33, 385, 800][seed % 6])
    group, kv_heads, page = int(rng.choice([1, 3, 4, 32, 128])), int(rng.integers(1, 5)), int(rng.choice([16, 64, 128, 1024]))
    nq = rng.integers(0, [4, 4, 40, 300][seed % 4], n) if seed % 2 or seed == 10 else np.ones(n, int)
    nq[0] = max(nq[0], 1)
    cuts = np.sort(rng.integers(0, n + 1, int(rng.integers(1, 6)))) if seed % 3 else np.array([0, n])
    shared = rng.integers(0, 5000, len(cuts) - 1)
    shared[rng.random(len(shared)) < 0.2] = 0
    part = np.zeros(n, int)
    for g, s in enumerate(shared):
        part[cuts[g]:cuts[g + 1]] = s
    own = np.maximum(rng.integers(0, 700, n), nq)
    kv_len = part + own
    out, err, share, n_q = _walk(lib, grid, nq, kv_len, cuts, shared, kv_heads, group, page)
    assert err == 0
    assert np.array_equal(out, _walk(lib, grid, nq, kv_len, cuts, shared, kv_heads, group, page, counted=1)[0])
    pack = _pack(int(max(nq)), group)
    items = _check(out, share, grid, _bounds(n_q, n, len(shared), kv_heads, group, pack))
    tile_q = 128 // group
    want = {}
    for g, s in enumerate(shared):
        tiles = -(-int(nq[cuts[g]:cuts[g + 1]].sum()) // tile_q)
        for i in range((tiles + 1) // 2 * kv_heads if s else 0):
            want[0, g, i] = -(-int(s) // 128)
    pieces = np.where(nq > 0, -(-(kv_len - part // 16 * 16) // 16), 0)
    for k in range(-(-n // pack)):
        mine = slice(k * pack, (k + 1) * pack)
        tiles = 1 if pack > 1 and nq[mine].sum() else -(-int(nq[mine].sum()) // tile_q)
        for i in range(tiles * kv_heads):
            want[1, k, i] = -(-int(pieces[mine].sum()) // 8)
    assert {k: v[0][6] for k, v in items.items()} == {k: v for k, v in want.items() if v > 0}


@pytest.mark.parametrize("bad", [dict(q_start=[0, 5, 2, 9, 12]), dict(q_start=[-3, 1, 2, 3, 40]), dict(q_start=[9, 9, 0, 3, 12]),
                                 dict(kv_len=[500, 10 ** 9, -5, 3]), dict(groups=[0, 3, 1]), dict(groups=[-2, 2, 9]),
                                 dict(shared=[10 ** 9, 100]), dict(shared=[-1, 100]), dict(max_q=2)])
def test_offsets_that_contradict_each_other_stay_inside(lib, bad):
    a = dict(nq=[3, 3, 3, 3], kv_len=[500, 400, 300, 450], groups=[0, 2, 4], shared=[200, 100], kv_heads=2, group=4, page=16, width=40,
             n_q=12)
    assert _walk(lib, 13, **a)[1] == 0
    out, err, share, n_q = _walk(lib, 13, **{**a, **bad})
    assert err == 1
    again = _walk(lib, 13, **{**a, **bad}, counted=1)
    assert np.array_equal(out, again[0]) and again[1] == 1
    bound = _bounds(12, 4, 2, 2, 4, _pack(bad.get("max_q", 3), 4))
    assert all(0 <= r[7] < bound[r[0]] and r[3] < r[4] for r in out.tolist())


def test_no_work(lib):
    out, err, share, n_q = _walk(lib, 20, [0, 0, 1], [5, 0, 0], [0, 3], [0], 2, 4, 16, n_q=1, max_q=1)
    assert len(out) == 0 and err == 0


@pytest.mark.parametrize("n,n_groups", [(400, 1500), (5000, 0), (2500, 400), (769, 1), (770, 385)])
def test_many_sequences_and_groups(lib, n, n_groups):
    rng = np.random.default_rng(n)
    nq = rng.integers(0, 3, n)
    cuts = np.sort(np.concatenate([[0], rng.integers(0, n + 1, max(0, n_groups - 1)), [n]])) if n_groups else np.array([0])
    shared = rng.integers(0, 300, n_groups)
    part = np.zeros(n, int)
    for g, s in enumerate(shared):
        part[cuts[g]:cuts[g + 1]] = s
    kv_len = part + np.maximum(rng.integers(0, 100, n), nq)
    out, err, share, n_q = _walk(lib, 19, nq, kv_len, cuts, shared, 2, 4, 16)
    assert err == 0
    items = _check(out, share, 19, _bounds(n_q, n, n_groups, 2, 4, _pack(2, 4)))
    with_keys = {(0, g, i) for g, s in enumerate(shared) if s for i in range(2 * (-(-int(nq[cuts[g]:cuts[g + 1]].sum()) // 32)))}
    packs = _pack(2, 4)
    pieces = np.where(nq > 0, -(-(kv_len - part // 16 * 16) // 16), 0)
    with_keys |= {(1, k, i) for k in range(-(-n // packs)) if pieces[k * packs:(k + 1) * packs].sum() for i in range(2)}
    # (two tiles of a group are one item)
    assert {k for k in items if k[0]} == {k for k in with_keys if k[0]} and {k for k in items if not k[0]} <= {k for k in with_keys if not k[0]}
    assert {k[:2] for k in items} == {k[:2] for k in with_keys}
