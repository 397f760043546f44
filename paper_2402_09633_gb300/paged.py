"""Several hypotheses of a sequence: caches in pages, attention that reads what hypotheses share once, the choice of the
best continuations, and moving states to them (ctypes binding of the same calls in include/gnn.h; argument marshalling
only)."""
from __future__ import annotations

import ctypes
import math
import struct

from . import binding
from . import sequence as Q
from .binding import GNN_OK, GnnError

_vp, _i64, _i32, _f32, _u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_uint64


class GnnPages(ctypes.Structure):
    _fields_ = [("k", Q.GnnHeads), ("v", Q.GnnHeads), ("n_pages", _i64), ("dtype", _i32), ("head_dim", _i32),
                ("page_size", _i32), ("table_width", _i32), ("table", _vp), ("table_stride", _i64), ("kv_len", _vp),
                ("n_seqs", _i32), ("reserved", _i32), ("status", _vp)]


class GnnAppendCall(ctypes.Structure):
    _fields_ = [("q", Q.GnnHeads), ("k", Q.GnnHeads), ("v", Q.GnnHeads), ("q_out", Q.GnnHeads), ("q_gain", _vp),
                ("k_gain", _vp), ("positions", _vp), ("q_start", _vp), ("n_rows", _i64), ("eps", _f32),
                ("positions_float", _i32)]


class GnnPagedCall(ctypes.Structure):
    _fields_ = [("q", Q.GnnHeads), ("out", Q.GnnHeads), ("q_start", _vp), ("group_start", _vp), ("shared_len", _vp),
                ("n_q_rows", _i64), ("n_groups", _i32), ("max_q", _i32), ("scale", _f32), ("reserved", _i32),
                ("workspace", _vp), ("workspace_bytes", _u64)]


class GnnBeamCall(ctypes.Structure):
    _fields_ = [("logits", _vp), ("row_stride", _i64), ("n_groups", _i64), ("scores", _vp), ("ended", _vp), ("dtype", _i32),
                ("beams", _i32), ("vocab", _i32), ("best", _i32), ("end_token", _i32), ("reserved", _i32),
                ("out_scores", _vp), ("out_parents", _vp), ("out_tokens", _vp), ("workspace", _vp), ("workspace_bytes", _u64)]


class GnnBeamState(ctypes.Structure):
    _fields_ = [("data", _vp), ("out", _vp), ("stride", _i64), ("out_stride", _i64), ("row_bytes", _i64)]


_H = "PqqiI"
_PAGES = struct.Struct(_H * 2 + "qiiiiPqPiIP").pack
_APPEND = struct.Struct(_H * 4 + "PPPPqfi").pack
_ATTEND = struct.Struct(_H * 2 + "PPPqiifiPQ").pack
_BEAM = struct.Struct("PqqPPiiiiiIPPPPQ").pack
_STATE = struct.Struct("PPqqq").pack
assert struct.calcsize(_H * 2 + "qiiiiPqPiIP") == ctypes.sizeof(GnnPages)
assert struct.calcsize(_H * 4 + "PPPPqfi") == ctypes.sizeof(GnnAppendCall)
assert struct.calcsize(_H * 2 + "PPPqiifiPQ") == ctypes.sizeof(GnnPagedCall)
assert struct.calcsize("PqqPPiiiiiIPPPPQ") == ctypes.sizeof(GnnBeamCall)
assert struct.calcsize("PPqqq") == ctypes.sizeof(GnnBeamState)
_NONE = (0, 0, 0, 0, 0)                                    # no view
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = Q._library()
        i = ctypes.c_int
        lib.gnn_paged_append.argtypes = [_vp, _vp, _vp, _vp]
        lib.gnn_paged_workspace.argtypes = [_vp, _vp, _vp]
        lib.gnn_paged_attend.argtypes = [_vp, _vp, _vp]
        lib.gnn_beam_workspace.argtypes = [_vp, _vp]
        lib.gnn_beam_select.argtypes = [_vp, _vp]
        lib.gnn_beam_reorder.argtypes = [_vp, _i64, i, _vp, i, _vp]
        lib.gnn_paged_reorder.argtypes = [_vp, i, _vp, _i64, i, _vp]
        for f in (lib.gnn_paged_append, lib.gnn_paged_workspace, lib.gnn_paged_attend, lib.gnn_beam_workspace, lib.gnn_beam_select,
                  lib.gnn_beam_reorder, lib.gnn_paged_reorder):
            f.restype = i
        waits = binding.load_library()                       # waits for the stream, without the interpreter lock
        waits.gnn_paged_status.argtypes = [_vp, _vp]
        waits.gnn_paged_status.restype = i
        _lib = lib
    return _lib


def _check(rc, what):
    if rc != GNN_OK:
        raise GnnError(rc, what)


_sizes = {}                                                # workspace bytes of calls, by what they depend on


def _workspace(key, ask, device, stream):
    """Memory for a call whose size `ask(address)` of the library says; the same sizes are asked for once."""
    n = _sizes.get(key)
    if n is None:
        size = _u64()
        ask(ctypes.byref(size))
        if len(_sizes) >= 4096:
            _sizes.clear()
        n = _sizes[key] = size.value
    return _empty(n, Q._torch.uint8, device, stream), n


def _empty(n, dtype, device, stream):
    """Memory of the call's stream: what another stream's held before may still be in use there."""
    torch = Q._torch
    if stream is None:
        return torch.empty(n, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=dtype, device=device)


class PagedCache:
    """Keys and values of sequences in pages, k and v [pages * page_size, heads, dim] (views, last stride 1): position j of
    sequence b lies in row table[b, j // page_size] * page_size + j % page_size.  table: cuda int32 [sequences, entries], last
    stride 1; kv_len: cuda int32 [sequences].  The tensors are the caller's, and the caller changes them (a step adds
    to kv_len what it is about to append).  Caches of several layers may have one table and kv_len.  What calls find out of
    range is in status().  The constructor waits for the current stream."""

    def __init__(self, k, v, table, kv_len, page_size: int):
        lib = _library()
        dtype, number, device, dim = Q._kind(k)
        assert k.shape[0] == v.shape[0] and k.shape[0] % page_size == 0, "k and v are whole pages, as many of each"
        assert table.dim() == 2 and table.get_device() == device and table.dtype == Q._torch.int32 and \
            (table.stride(1) == 1 or table.shape[1] == 1), "table: cuda int32 [sequences, entries], last stride 1"
        n = table.shape[0]
        self.kv_len_at = Q._vector(kv_len, n, Q._torch.int32, device)
        self.k, self.v, self.table, self.kv_len, self.page_size = k, v, table, kv_len, page_size
        self.dtype, self.device, self.dim, self.lib = dtype, device, dim, lib
        self.shape = dim, page_size, table.shape, k.shape[1]                     # what sizes depend on
        self.word = Q._torch.zeros(1, dtype=Q._torch.int32, device=k.device)
        Q._torch.cuda.current_stream().synchronize()         # the zero is there before any stream's first call
        self.pages = _PAGES(*Q._fields(k, dtype, device, dim), *Q._fields(v, dtype, device, dim), k.shape[0] // page_size, number,
                            dim, page_size, table.shape[1], table.data_ptr(), table.stride(0), self.kv_len_at or 0, n, 0,
                            self.word.data_ptr())

    def _starts(self, q_start):
        return Q._vector(q_start, self.table.shape[0] + 1, Q._torch.int32, self.device)

    def append(self, rot, q_start, k, v, q=None, positions=None, q_gain=None, k_gain=None, eps=None, q_out=None, stream=None):
        """New rows k, v [rows, heads, dim] into their pages, k rotated by rot (a Rotary), normalised before with eps: rows
        q_start[b] .. q_start[b + 1] - 1 are the last positions of sequence b.  q, when given, is rotated (and
        normalised) into q_out, which is returned.  positions: as for rope, None: those in the sequences."""
        device, dtype, dim = self.device, self.dtype, self.dim
        assert Q._current_device() == device, "the cache's device is not the current one"
        n = k.shape[0]
        assert v.shape == k.shape and k.shape[1] == self.k.shape[1], "k and v of other sizes than the cache's"
        queries = queries_out = _NONE
        if q is not None:
            assert q.shape[0] == n, "as many queries as keys"
            if q_out is None:
                q_out = Q._empty_like(q, stream)
            assert q_out.shape == q.shape
            queries, queries_out = Q._fields(q, dtype, device, dim), Q._fields(q_out, dtype, device, dim)
        else:
            assert q_out is None, "q_out without q"
        assert eps is None or eps > 0, "eps: above zero, or None: no norms"
        pos, real = Q._positions(positions, n, device)
        f32 = Q._torch.float32
        if n == 0 or self.table.shape[0] == 0:
            return q_out
        call = _APPEND(*queries, *Q._fields(k, dtype, device, dim), *Q._fields(v, dtype, device, dim), *queries_out,
                       Q._vector(q_gain, dim, f32, device) or 0, Q._vector(k_gain, dim, f32, device) or 0, pos or 0,
                       self._starts(q_start), n, eps or 0.0, real)
        _check(self.lib.gnn_paged_append(self.pages, rot.address, call, Q._stream(stream, device)), "gnn_paged_append")
        return q_out

    def attend(self, q, q_start, groups=None, shared=None, scale=None, max_q: int = 0, out=None, stream=None):
        """Attention of q [rows, heads, dim]: row i of the nq rows q_start[b] .. q_start[b + 1] - 1 sees sequence b's keys up to
        its own position kv_len[b] - nq + i.  groups: cuda int32 [groups + 1], shared: cuda int32 [groups]: sequences
        groups[g] .. groups[g + 1] - 1 have their first shared[g] positions in common, which are read once, through the
        first one's pages.  max_q: the most queries of a sequence, when known: short sequences are computed together only then."""
        device, dtype, dim = self.device, self.dtype, self.dim
        assert Q._current_device() == device, "the cache's device is not the current one"
        assert (groups is None) == (shared is None), "groups and shared go together"
        if out is None:
            out = Q._empty_like(q, stream)
        assert out.shape == q.shape, "out of another size"
        n = q.shape[0]
        if n == 0 or self.table.shape[0] == 0:
            return out
        n_groups, int32 = 0 if groups is None else shared.numel(), Q._torch.int32
        where = (Q._vector(groups, n_groups + 1, int32, device), Q._vector(shared, n_groups, int32, device)) if n_groups else (0, 0)
        fields = (*Q._fields(q, dtype, device, dim), *Q._fields(out, dtype, device, dim), self._starts(q_start), *where, n, n_groups,
                  max_q, 1.0 / math.sqrt(dim) if scale is None else scale, 0)
        lib = self.lib
        space, size = _workspace((device, self.shape, q.shape[1], n, n_groups, max_q),
                                 lambda at: _check(lib.gnn_paged_workspace(self.pages, _ATTEND(*fields, 0, 0), at), "gnn_paged_workspace"),
                                 device, stream)
        rc = lib.gnn_paged_attend(self.pages, _ATTEND(*fields, space.data_ptr(), size), Q._stream(stream, device))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_paged_attend")
        return out

    def status(self, stream=None) -> int:
        return binding.load_library().gnn_paged_status(self.word.data_ptr(), binding._stream_handle(stream))


def beam_select(logits, scores, beams: int, best=None, ended=None, end: int = 0, stream=None):
    """(scores, parents, tokens), each [groups * best]: of every group of `beams` rows of logits [rows, vocab] (last stride 1)
    with their scores (cuda float32 [rows]), the best continuations in order, valued score + log-probability; parents are
    rows within the group.  ended (cuda bool or uint8 [rows]): rows whose one continuation is `end` at their score.  best:
    beams, unless given.  Where there are fewer, -inf, 0, -1."""
    lib = _library()
    device, torch = logits.get_device(), Q._torch
    assert device >= 0 and device == Q._current_device(), "a cuda tensor of the current device"
    assert logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1), "logits [rows, vocab], last stride 1"
    assert logits.dtype in Q.DTYPES, f"type {logits.dtype} is not taken"
    rows, vocab = logits.shape
    assert beams >= 1 and rows % beams == 0, "rows are whole groups of beams"
    groups, best = rows // beams, beams if best is None else best
    if ended is not None:
        assert ended.dtype in (torch.bool, torch.uint8), "ended: bool or uint8"
    dtype = Q.DTYPES[logits.dtype]
    at = Q._vector(scores, rows, torch.float32, device), Q._vector(ended, rows, None if ended is None else ended.dtype, device) or 0
    size = max(0, groups * best)
    out, parents = _empty(size, torch.float32, device, stream), _empty(size, torch.int32, device, stream)
    tokens = _empty(size, torch.int32, device, stream)
    if rows == 0:
        return out, parents, tokens
    fields = (logits.data_ptr(), logits.stride(0), groups, *at, dtype, beams, vocab, best, end, 0, out.data_ptr(), parents.data_ptr(),
              tokens.data_ptr())
    space, n = _workspace((device, dtype, groups, beams, vocab, best),
                          lambda at: _check(lib.gnn_beam_workspace(_BEAM(*fields, 0, 0), at), "gnn_beam_workspace"), device, stream)
    rc = lib.gnn_beam_select(_BEAM(*fields, space.data_ptr(), n), Q._stream(stream, device))
    if rc != GNN_OK:
        raise GnnError(rc, "gnn_beam_select")
    return out, parents, tokens


def _state(x, y, rows, device):
    shape = x.shape
    assert x.get_device() == device and shape[0] == rows, "states: cuda tensors [rows, ...] of the parents' device"
    assert y is x or (y.get_device() == device and y.shape == shape and y.dtype == x.dtype), "out: tensors like the states"
    whole = x.nbytes
    if whole == 0:
        return _STATE(0, 0, 0, 0, 0)
    inner = whole // rows
    strides = [_row_stride(x, inner), inner]
    strides[1] = strides[0] if y is x else _row_stride(y, inner)
    return _STATE(x.data_ptr(), y.data_ptr(), *strides, inner)


def _row_stride(x, inner):
    """Bytes from a row to the next."""
    if x.is_contiguous():
        return inner
    stride = x.stride(0) * x.element_size()
    assert x[0].is_contiguous(), "a state's row is contiguous"
    assert stride >= inner or x.shape[0] == 1, "rows overlap"
    return max(stride, inner)


def beam_reorder(parents, beams: int, states=(), out=None, caches=(), stream=None):
    """States of hypotheses moved to those that continue them: row i of a group of `beams` rows of each tensor of `states`
    [rows, ...] gets what row parents[i] of the group held (parents: cuda int32 [rows]), in place or, with `out`, in
    tensors like them.  caches: PagedCaches with one table and kv_len, whose sequences are the rows, always in place: full pages
    are shared with the parent, the rows of the page that it has begun are copied (see gnn_paged_reorder).  Where a state or a
    cache is refused, nothing moves.  Returns the states' new tensors."""
    lib = _library()
    device, rows = parents.get_device(), parents.numel()
    assert device >= 0 and device == Q._current_device(), "a cuda tensor of the current device"
    assert beams >= 1 and rows % beams == 0, "rows are whole groups of beams"
    at, st = Q._vector(parents, rows, Q._torch.int32, device), Q._stream(stream, device)
    states, caches = list(states), list(caches)
    new = states if out is None else list(out)
    assert len(new) == len(states), "as many outputs as states"
    moves = b"".join([_state(x, y, rows, device) for x, y in zip(states, new)])
    for c in caches:
        assert c.device == device and c.table.shape[0] == rows, "caches of as many sequences, on the same device"
    if rows == 0:
        return new
    if caches:                                               # nothing moves unless both calls are taken: the states' as one of no groups first
        if states:
            _check(lib.gnn_beam_reorder(at, 0, beams, moves, len(new), st), "gnn_beam_reorder")
        _check(lib.gnn_paged_reorder(b"".join([c.pages for c in caches]), len(caches), at, rows // beams, beams, st),
               "gnn_paged_reorder")
    if states:
        _check(lib.gnn_beam_reorder(at, rows // beams, beams, moves, len(new), st), "gnn_beam_reorder")
    return new
