"""The sequence binding called by several threads at once (no GPU): a stand-in library, called the same way, checks that
each call gets its own arguments."""
import ctypes
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2402_09633_gb300 import binding
from paper_2402_09633_gb300 import sequence as Q

# Every address of call `id` is id << 20 plus the argument's own number, and its counts are id.
STAND_IN = r"""
#include "gnn.h"
static int at(const void* p, int64_t id, int what) { return (int64_t)p == (id << 20) + what; }
static int view(const gnn_heads* h, int64_t id, int what) {
  return at(h->data, id, what) && h->row_stride == 64 * id && h->head_stride == 64 && h->n_heads == 1 && h->reserved == 0;
}
int gnn_rotary_init(const gnn_rotary_config* c, gnn_rotary* out) { return c && out ? GNN_OK : GNN_ERR_INVALID_ARG; }
int gnn_rope(const gnn_rotary* rot, int dtype, int dim, const gnn_heads* x, const gnn_heads* y, const void* pos,
             int real, int64_t n, gnn_stream_t stream) {
  return rot && dtype == 1 && dim == 64 && !real && view(x, n, 1) && view(y, n, 2) && at(pos, n, 3) && at(stream, n, 4)
      ? GNN_OK : GNN_ERR_INVALID_ARG;
}
int gnn_qk_norm_rope(const gnn_rotary* rot, int dtype, int dim, float eps, const float* gq, const float* gk,
                     const gnn_heads* q, const gnn_heads* k, const gnn_heads* v, const gnn_heads* qo,
                     const gnn_heads* ko, const gnn_heads* vo, const void* pos, int real, const int64_t* rows,
                     int64_t out_rows, int64_t n, gnn_stream_t stream) {
  return rot && dtype == 1 && dim == 64 && eps > 0 && !gq && !gk && view(q, n, 1) && view(k, n, 2) &&
         (n % 2 ? !v && !vo : view(v, n, 3) && view(vo, n, 6)) && view(qo, n, 4) && view(ko, n, 5) && at(pos, n, 7) &&
         !real && at(rows, n, 8) && out_rows == n && at(stream, n, 9) ? GNN_OK : GNN_ERR_INVALID_ARG;
}
int gnn_attention_create(gnn_attention** out) { *out = (gnn_attention*)out; return GNN_OK; }
int gnn_attention_status(gnn_attention* a, gnn_stream_t stream) { return a ? GNN_OK : GNN_ERR_INVALID_ARG; }
void gnn_attention_destroy(gnn_attention* a) {}
int gnn_attention_run(gnn_attention* a, const gnn_attention_call* c, gnn_stream_t stream) {
  int64_t n = c->n_q_rows;
  return a && c->dtype == 1 && c->head_dim == 64 && view(&c->q, n, 1) && view(&c->k, n, 2) && view(&c->v, n, 3) &&
         view(&c->out, n, 4) && at(c->q_start, n, 5) && at(c->kv_start, n, 6) && at(c->kv_len, n, 7) && c->n_kv_rows == n &&
         c->n_seqs == 1 && c->max_q == n && c->max_kv == n && c->left == n && c->right == 0 && c->sinks == 3 &&
         c->scale == 0.125f && c->reserved == 0 && at(stream, n, 8) ? GNN_OK : GNN_ERR_INVALID_ARG;
}
"""


class Tensor:
    """What the binding asks of a cuda tensor, without memory behind it."""
    device = 0

    def __init__(self, address, dtype, *shape):
        self.address, self.dtype, self.shape = address, dtype, shape

    def stride(self):
        return (64 * self.shape[0], 64, 1)

    def get_device(self):
        return self.device

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.shape[0]

    def is_contiguous(self):
        return True


class Stream:
    def __init__(self, address):
        self.cuda_stream = address


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    where = tmp_path_factory.mktemp("stand_in")
    (where / "lib.c").write_text(STAND_IN)
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(binding.__file__))), "include")
    lib = str(where / "lib.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I", include, "-o", lib, str(where / "lib.c")], check=True)
    return lib


@pytest.fixture
def patched(stand_in, monkeypatch):
    Q._library()                                             # the real one, whose place is given back afterwards
    monkeypatch.setattr(Q, "_lib", None)
    monkeypatch.setattr(binding, "LIB_PATH", stand_in)
    monkeypatch.setattr(binding, "_lib", ctypes.CDLL(stand_in))
    Q._library()
    monkeypatch.setattr(Q, "_current_device", lambda: Tensor.device)
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    yield
    sys.setswitchinterval(interval)


def _calls(kind, n, attend):
    bf16, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    head = lambda what: Tensor((n << 20) + what, bf16, n, 1, 64)                       # noqa: E731
    vector = lambda what, dtype=i32, m=n: Tensor((n << 20) + what, dtype, m)           # noqa: E731
    stream = lambda what: Stream((n << 20) + what)                                     # noqa: E731
    if kind == "rope":
        rot = Q.Rotary(64)
        return lambda: Q.rope(rot, head(1), vector(3), out=head(2), stream=stream(4))
    if kind == "norm":
        rot = Q.Rotary(64)
        v, v_out = (None, None) if n % 2 else (head(3), head(6))
        return lambda: Q.qk_norm_rope(rot, head(1), head(2), vector(7), v=v, q_out=head(4), k_out=head(5), v_out=v_out,
                                      rows=vector(8, i64), stream=stream(9))
    return lambda: attend(head(1), head(2), head(3), vector(5, i32, 2), left=n, right=0, sinks=3, kv_start=vector(6, i32, 1),
                          kv_len=vector(7, i32, 1), max_q=n, max_kv=n, out=head(4), stream=stream(8))


@pytest.mark.parametrize("kinds", [("rope",), ("norm",), ("attend",), ("rope", "norm", "attend")])
def test_each_call_gets_its_own_arguments(patched, kinds):
    wrong, done = [], []

    def work(n):
        attend = Q.WindowAttention()
        call = _calls(kinds[n % len(kinds)], n, attend)
        for _ in range(12000):
            try:
                call()
            except Exception as e:                           # refused: not what this thread gave it
                wrong.append((n, repr(e)))
        attend.close()
        done.append(n)

    threads = [threading.Thread(target=work, args=(n,)) for n in range(2, 8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(done) == 6
    assert not wrong, f"{len(wrong)} of {6 * 12000} calls got another's arguments, or none: {wrong[:3]}"
