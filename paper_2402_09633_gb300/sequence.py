"""Hits read as a sequence: rotary positions, norms of queries and keys with the rotation, and attention with a
sliding window (ctypes binding of the same calls in include/gnn.h; argument marshalling only).

All tensors are views [rows, heads, head_dim] on the GPU whose last stride is 1, so slices of a packed projection
are taken as they are."""
from __future__ import annotations

import ctypes
import math

from . import binding
from .binding import GNN_OK, GnnError, _stream_handle

DTYPES = {"torch.float32": 0, "torch.bfloat16": 1, "torch.float16": 2}
LAYOUTS = {"half": 0, "interleaved": 1}
_vp, _i64, _i32, _f32, _f64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_double


class GnnHeads(ctypes.Structure):
    _fields_ = [("data", _vp), ("row_stride", _i64), ("head_stride", _i64), ("n_heads", _i32), ("reserved", _i32)]


class GnnRotaryConfig(ctypes.Structure):
    _fields_ = [("rot_dim", _i32), ("layout", _i32), ("scaling", _i32), ("reserved", _i32), ("base", _f64),
                ("factor", _f64), ("length", _f64), ("slow", _f64), ("fast", _f64), ("amplitude", _f64)]


class GnnRotary(ctypes.Structure):
    _fields_ = [("rot_dim", _i32), ("layout", _i32), ("amplitude", _f32), ("magic", _i32),
                ("turn_fixed", ctypes.c_uint64 * 128), ("turn_hi", _f32 * 128), ("turn_lo", _f32 * 128)]


class GnnAttentionCall(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("head_dim", _i32), ("q", GnnHeads), ("k", GnnHeads), ("v", GnnHeads),
                ("out", GnnHeads), ("q_start", _vp), ("kv_start", _vp), ("kv_len", _vp), ("n_q_rows", _i64),
                ("n_kv_rows", _i64), ("n_seqs", _i32), ("max_q", _i32), ("max_kv", _i32), ("left", _i32),
                ("right", _i32), ("sinks", _i32), ("scale", _f32), ("reserved", _i32)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        heads = ctypes.POINTER(GnnHeads)
        rot = ctypes.POINTER(GnnRotary)
        i = ctypes.c_int
        lib.gnn_rotary_init.argtypes = [ctypes.POINTER(GnnRotaryConfig), rot]
        lib.gnn_rope.argtypes = [rot, i, i, heads, heads, _vp, i, _i64, _vp]
        lib.gnn_qk_norm_rope.argtypes = [rot, i, i, _f32, _vp, _vp, heads, heads, heads, heads, heads, heads, _vp, i,
                                         _vp, _i64, _i64, _vp]
        lib.gnn_attention_create.argtypes = [ctypes.POINTER(_vp)]
        lib.gnn_attention_run.argtypes = [_vp, ctypes.POINTER(GnnAttentionCall), _vp]
        lib.gnn_attention_status.argtypes = [_vp, _vp]
        for f in (lib.gnn_rotary_init, lib.gnn_rope, lib.gnn_qk_norm_rope, lib.gnn_attention_create,
                  lib.gnn_attention_run, lib.gnn_attention_status):
            f.restype = i
        lib.gnn_attention_destroy.argtypes = [_vp]
        lib.gnn_attention_destroy.restype = None
        _lib = lib
    return _lib


def _heads(x, like=None):
    """A view's struct; x: cuda tensor [rows, heads, dim], last stride 1."""
    assert x.is_cuda and x.dim() == 3 and (x.stride(2) == 1 or x.shape[2] == 1), "a cuda tensor [rows, heads, dim], last stride 1"
    if like is not None:
        assert x.dtype == like.dtype and x.device == like.device and x.shape[2] == like.shape[2], "types, devices or head sizes differ"
    return GnnHeads(x.data_ptr(), x.stride(0), x.stride(1), x.shape[1], 0)


def _dtype(x):
    d = DTYPES.get(str(x.dtype))
    assert d is not None, f"type {x.dtype} is not taken"
    return d


def _vector(x, n, dtype, device):
    """A contiguous cuda vector's address, or None."""
    if x is None:
        return None
    assert x.device == device and x.dtype == dtype and x.is_contiguous() and x.numel() == n, \
        f"a contiguous {dtype} cuda tensor of {n} is wanted"
    return x.data_ptr()


def _positions(pos, n, device):
    import torch
    if pos is None:
        return None, 0
    real = pos.dtype == torch.float32
    return _vector(pos, n, torch.float32 if real else torch.int32, device), int(real)


class Rotary:
    """The table of a rotation.  scaling: None, ("linear", factor) or ("turns", factor, length, slow, fast); see
    gnn_rotary_init in include/gnn.h."""

    def __init__(self, rot_dim: int, base: float = 10000.0, layout: str = "half", scaling=None, amplitude: float = 1.0):
        kind, *args = scaling or ("plain",)
        kinds = {"plain": (0, 0), "linear": (1, 1), "turns": (2, 4)}
        assert layout in LAYOUTS, f"layout {layout!r}"
        assert kind in kinds and len(args) == kinds[kind][1], f"scaling {scaling!r}"
        args = [float(a) for a in args] + [0.0] * (4 - len(args))
        cfg = GnnRotaryConfig(rot_dim, LAYOUTS[layout], kinds[kind][0], 0, base, *args, amplitude)
        self.table = GnnRotary()
        rc = _library().gnn_rotary_init(ctypes.byref(cfg), ctypes.byref(self.table))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_rotary_init")
        self.ref = ctypes.byref(self.table)


def rope(rot: Rotary, x, positions=None, out=None, stream=None):
    """x [rows, heads, dim] rotated by positions (cuda int32 or float32 [rows]; None: row numbers).  out may be x."""
    import torch
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    assert out.shape == x.shape
    pos, real = _positions(positions, x.shape[0], x.device)
    if x.shape[0] == 0:
        return out
    rc = _library().gnn_rope(rot.ref, _dtype(x), x.shape[2], ctypes.byref(_heads(x)), ctypes.byref(_heads(out, x)), pos,
                             real, x.shape[0], _stream_handle(stream))
    if rc != GNN_OK:
        raise GnnError(rc, "gnn_rope")
    return out


def qk_norm_rope(rot: Rotary, q, k, positions=None, v=None, q_gain=None, k_gain=None, eps: float = 1e-6, q_out=None,
                 k_out=None, v_out=None, rows=None, stream=None):
    """(q_out, k_out, v_out): q and k normalised for each head and rotated, v copied.  With rows (cuda int64 [rows]),
    row r of k and v goes to row rows[r] of k_out and v_out, which are then given."""
    import torch
    n = q.shape[0]
    assert k.shape[0] == n and (v is None or v.shape == k.shape)
    assert rows is None or (k_out is not None and (v is None or v_out is not None)), "rows need k_out and v_out"
    assert v is not None or v_out is None, "v_out without v"
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
    if v is not None and v_out is None:
        v_out = torch.empty(v.shape, dtype=v.dtype, device=v.device)
    assert q_out.shape == q.shape and k_out.shape[1:] == k.shape[1:] and (rows is not None or k_out.shape[0] == n)
    assert v is None or (v_out.shape[1:] == v.shape[1:] and v_out.shape[0] == k_out.shape[0])
    pos, real = _positions(positions, n, q.device)
    at = _vector(rows, n, torch.int64, q.device)
    gains = [_vector(g, q.shape[2], torch.float32, q.device) for g in (q_gain, k_gain)]
    if n == 0 or k_out.shape[0] == 0:
        assert n == 0, "k_out has no rows"
        return q_out, k_out, v_out
    views = [None if x is None else ctypes.byref(_heads(x, q)) for x in (q, k, v, q_out, k_out, v_out)]
    rc = _library().gnn_qk_norm_rope(rot.ref, _dtype(q), q.shape[2], eps, *gains, *views, pos, real, at,
                                     k_out.shape[0], n, _stream_handle(stream))
    if rc != GNN_OK:
        raise GnnError(rc, "gnn_qk_norm_rope")
    return q_out, k_out, v_out


class WindowAttention:
    """One handle of gnn_attention_create on the current device (a stream's own; see include/gnn.h)."""

    def __init__(self):
        self.lib = _library()
        h = _vp()
        rc = self.lib.gnn_attention_create(ctypes.byref(h))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_attention_create")
        self.handle = h

    def __call__(self, q, k, v, q_start, left: int = -1, right: int = -1, sinks: int = 0, scale=None, kv_start=None,
                 kv_len=None, max_q: int = 0, max_kv: int = 0, out=None, stream=None):
        """Attention of the queries q [rows, heads, dim] over the keys and values k, v [kv rows, kv heads, dim], bf16 or
        fp16.  q_start: cuda int32 [sequences + 1]; kv_start, kv_len: cuda int32 [sequences], or None: a sequence's keys
        are the rows of its queries.  left, right: keys visible before and after a query's own position (-1: all),
        sinks: first keys that stay visible; max_q, max_kv: the most queries and keys of a sequence, when known."""
        import torch
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        n = q_start.numel() - 1
        assert n >= 0 and out.shape == q.shape and k.shape == v.shape
        call = GnnAttentionCall(_dtype(q), q.shape[2], _heads(q), _heads(k, q), _heads(v, q), _heads(out, q),
                                _vector(q_start, n + 1, torch.int32, q.device), _vector(kv_start, n, torch.int32, q.device),
                                _vector(kv_len, n, torch.int32, q.device), q.shape[0], k.shape[0], n, max_q, max_kv, left,
                                right, sinks, 1.0 / math.sqrt(q.shape[2]) if scale is None else scale, 0)
        rc = self.lib.gnn_attention_run(self.handle, ctypes.byref(call), _stream_handle(stream))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_attention_run")
        return out

    def status(self, stream=None) -> int:
        return self.lib.gnn_attention_status(self.handle, _stream_handle(stream))

    def close(self):
        if getattr(self, "handle", None):
            self.lib.gnn_attention_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
