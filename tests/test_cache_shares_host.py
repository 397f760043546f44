"""How the attention over a cache shares out its units of keys (csrc/attend_few.cuh), run on the CPU from its own source:
every block takes as many, all are taken, and sums past 32 bits (sequences that read the same keys) stay what they are."""
import ctypes

import numpy as np
import pytest

from tests import host_cuda

MAIN = r"""
#include "ptx.cuh"
#include <cmath>
using std::max;
using std::min;
#include "shares.cuh"
using namespace gnn;
extern "C" long long shares(int n_seqs, const int* q_start, const int* kv_start, const int* kv_len, int n_q, int n_kv, int KR,
                            int grid, int sixteen, long long* pre, unsigned* err) {
  AttendParams p = {};
  p.q_start = q_start; p.kv_start = kv_start; p.kv_len = kv_len;
  p.n_q_rows = n_q; p.n_kv_rows = n_kv; p.n_seqs = n_seqs; p.max_q = n_q;
  p.left = -1; p.right = 0;
  p.err = err;
  static int64_t all[kFewSeqs + 1];
  static uint32_t sums[kFewWarps];
  static Sequence first[32 * kFewWarps];
  long long share = -1;
  host::launch(grid, 32 * kFewWarps, [&] {
    if (blockIdx.x) return;
    const int64_t s = sixteen ? few_share<2>(p, KR, all, sums, first) : few_share<1>(p, KR, all, sums, first);
    if (threadIdx.x == 0) share = s;
  });
  for (int b = 0; b <= n_seqs; ++b) pre[b] = all[b];
  return share;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cut = host_cuda.between
    text = "namespace gnn {\n"
    text += cut(host_cuda.source("rotary.cuh"), "struct HeadsView {", "struct RotaryParams {")
    text += cut(host_cuda.source("attend.cuh"), "struct AttendParams {", "// One query row of one head")
    few = host_cuda.source("attend_few.cuh")
    text += cut(few, "constexpr int kFewWarps", "struct FewGrid {") + cut(few, "// Keys that some query", "// NC: 16-byte pieces")
    lib = host_cuda.compile_host(tmp_path_factory.mktemp("host"), MAIN, [("shares.cuh", text + "}\n")])
    vp, i = ctypes.c_void_p, ctypes.c_int
    lib.shares.argtypes = [i, vp, vp, vp, i, i, i, i, i, vp, vp]
    lib.shares.restype = ctypes.c_longlong
    return lib


MOST = 2147475455


@pytest.mark.parametrize("n_seqs,n_kv,low,KR,grid", [
    (1, 1028, 1028, 2, 34), (64, 8192, 4096, 4, 456), (128, 40, 1, 2, 256), (129, 3000, 1, 2, 456), (1024, 130, 0, 1, 456),
    (100, 16, 16, 2, 200), (7, 131072, 1, 3, 304), (128, MOST, MOST, 1, 456), (1024, MOST, MOST, 8, 304),
    (1024, 2 ** 27, 2 ** 27 - 5000, 1, 456), (70, MOST, 2 ** 30, 2, 456), (1024, MOST, MOST, 2 ** 14, 456)])
@pytest.mark.parametrize("sixteen", [0, 1])
def test_shares(lib, n_seqs, n_kv, low, KR, grid, sixteen):
    rng = np.random.default_rng(n_seqs)
    q_start = np.arange(n_seqs + 1, dtype=np.int32)
    kv_len = rng.integers(low, n_kv + 1, n_seqs, dtype=np.int64).astype(np.int32)
    kv_start = (n_kv - kv_len).astype(np.int32)
    pre, err = np.full(n_seqs + 1, -1, np.int64), np.zeros(1, np.uint32)
    at = lambda a: a.ctypes.data_as(ctypes.c_void_p)         # noqa: E731
    share = lib.shares(n_seqs, at(q_start), at(kv_start), at(kv_len), n_seqs, n_kv, KR, grid, sixteen, at(pre), at(err))
    units = np.maximum((kv_len.astype(np.int64) + 63) // 64, 1)
    taken = np.diff(pre)
    assert err[0] == 0 and pre[0] == 0 and share >= 1
    if np.array_equal(taken, units):
        least = int(np.sqrt(0.12 * (2 if sixteen else 1) * units.sum() / n_seqs))
        assert -(-int(units.sum()) * KR // grid) <= share <= max(-(-int(units.sum()) * KR // grid), least + 1)
    else:                                                    # small shares: every sequence's units fill whole ones
        assert share <= 16 and np.array_equal(taken, -(-units // share) * share)
    assert share * grid >= int(pre[-1]) * KR
