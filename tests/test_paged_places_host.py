"""Where the parts of the attention over pages leave their outputs (csrc/paged_tile.cuh), run on the CPU from its own source: apart
from each other, and inside a workspace of two places to a row and head and two to a thread block."""
import ctypes

import numpy as np
import pytest

from tests import host_cuda
from tests import test_paged_shares_host as S

# as the kernel does: every part's rows of both places
PART = r"""
      const int tile = own ? (int)e : 2 * (int)e, most = own ? g.box_b : g.box_a, have = w.nq - tile * g.tile_q;
      const long long at = paged_places(p, g, own, w.q0 + tile * g.tile_q, have, s % kv_heads) + (long long)blockIdx.x * 2 * (own ? g.rows_b : g.rows_a);
      const int rows0 = min(have, most) * g.group, rows1 = both ? min(have - g.tile_q, most) * g.group : rows0;
      const long long row[6] = {own, at, at + 2 * rows0 - 1, at + 1, at + 2 * rows1, n};        // every second row, from where to where
      for (int i = 0; i < 6; ++i) out[(long long)n * 6 + i] = row[i];
      ++n;
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cut, main = host_cuda.between, S.MAIN
    a = main.index("      const int64_t last = u0")
    main = main[:a] + PART + main[main.index("    };\n    paged_walk", a):]
    main = host_cuda.replace(main, "g.pack = pack;", "g.pack = pack; g.box_a = min(g.tile_q, n_q); g.box_b = min(g.tile_q, pack * min(max_q, n_q)); "
                             "g.rows_a = g.box_a * group; g.rows_b = g.box_b * group;")
    rotary, tile = host_cuda.source("rotary.cuh"), host_cuda.source("paged_tile.cuh")
    text = "namespace gnn {\n" + cut(rotary, "struct HeadsView {", "struct PagedPlace {")
    text += "constexpr int kTileQ = 128, kKeys = 128, kAttendThreads = 384;\n"
    text += cut(host_cuda.source("paged.cuh"), "struct PagedParams {", "// The row of position j")
    text += cut(tile, "constexpr int kPagedCost", "// A part of an item, as")
    text += "struct PagedBars { int64_t scan[2][12]; int64_t before; int at; PagedOwn own[kPagedKept]; PagedWork shared[kGroupsKept]; };\n"
    text += cut(tile, "// Block b's share of the list", "template <typename T, int DP>\n__global__")
    lib = host_cuda.compile_host(tmp_path_factory.mktemp("host"), main, [("shares.cuh", text + "}\n")])
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.walk.argtypes = [i] * 4 + [vp] * 4 + [i] * 6 + [vp, i, vp, vp, i]
    lib.walk.restype = i
    return lib


def _rows(lib, grid, nq, kv_len, cuts, shared, kv_heads, group, page, max_q, n_q=None, q_start=None, pack=None):
    i32 = lambda x: np.ascontiguousarray(x, dtype=np.int32)  # noqa: E731
    at = lambda a: a.ctypes.data_as(ctypes.c_void_p)         # noqa: E731
    q_start = i32(np.concatenate([[0], np.cumsum(nq)])) if q_start is None else i32(q_start)
    n_q = int(q_start[-1]) if n_q is None else n_q
    kv_len, cuts, shared = i32(kv_len), i32(cuts), i32(shared)
    known = max_q or n_q
    pack = S._pack(known, group)
    out, err, share = np.zeros((200000, 6), np.int64), np.zeros(1, np.uint32), np.zeros(1, np.int64)
    n = lib.walk(grid, n_q, kv_len.size, shared.size, at(q_start), at(kv_len), at(cuts), at(shared), known, kv_heads, group, pack, page,
                 -(-max(1, int(kv_len.max())) // page), at(out), len(out), at(err), at(share), 0)
    box = {0: min(128 // group, n_q), 1: min(128 // group, pack * min(known, n_q))}
    bound = {k: 2 * (n_q * kv_heads * group + grid * box[k] * group) for k in box}
    return out[:n], int(err[0]), bound


@pytest.mark.parametrize("known", [False, True])
@pytest.mark.parametrize("grid", [1, 7, 152])
@pytest.mark.parametrize("seed", range(10))
def test_parts_lie_apart(lib, grid, seed, known):
    rng = np.random.default_rng(seed)
    n = int([1, 3, 33, 385, 900][seed % 5])
    group, kv_heads, page = int(rng.choice([1, 3, 4, 25, 128])), int(rng.integers(1, 5)), int(rng.choice([16, 128]))
    nq = rng.integers(0, [3, 4, 40, 300][seed % 4], n) if seed % 2 else np.ones(n, int)
    nq[0] = max(nq[0], 1)
    cuts = np.sort(rng.integers(0, n + 1, int(rng.integers(1, 9)))) if seed % 3 else np.array([0, n])
    shared = rng.integers(0, 3000, len(cuts) - 1)
    part = np.zeros(n, int)
    for g, s in enumerate(shared):
        part[cuts[g]:cuts[g + 1]] = s
    kv_len = part + np.maximum(rng.integers(0, 500, n), nq)
    spare = int(rng.choice([0, 5]))                          # rows behind the last sequence
    out, err, bound = _rows(lib, grid, nq, kv_len, cuts, shared, kv_heads, group, page, int(max(nq)) if known else 0,
                            n_q=int(nq.sum()) + spare)
    assert err == 0 and len(out) > 0
    for own in (0, 1):
        rows = np.concatenate([np.arange(a, z, 2) for o, a0, z0, a1, z1, _ in out.tolist() if o == own for a, z in ((a0, z0), (a1, z1))] + [[]])
        assert len(np.unique(rows)) == len(rows) and (len(rows) == 0 or 0 <= rows.min() and rows.max() < bound[own])


@pytest.mark.parametrize("bad", [dict(q_start=[0, 5, 2, 9, 12]), dict(q_start=[-3, 1, 2, 3, 40]), dict(q_start=[9, 9, 0, 3, 12]),
                                 dict(kv_len=[500, 10 ** 9, -5, 3]), dict(cuts=[0, 3, 1]), dict(cuts=[-2, 2, 9]), dict(max_q=2), dict(max_q=1),
                                 dict(q_start=[0, 1, 2, 12, 12], max_q=1), dict(q_start=[0, 9, 10, 11, 12], max_q=1)])
def test_contradicting_offsets_stay_inside(lib, bad):
    a = dict(nq=[3, 3, 3, 3], kv_len=[500, 400, 300, 450], cuts=[0, 2, 4], shared=[200, 100], kv_heads=2, group=4, page=16, max_q=3, n_q=12)
    out, err, bound = _rows(lib, 13, **{**a, **bad})
    assert err == 1
    assert all(0 <= x <= bound[r[0]] for r in out.tolist() for x in r[1:5])
