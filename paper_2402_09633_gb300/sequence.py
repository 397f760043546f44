"""Hits read as a sequence: rotary positions, norms of queries and keys with the rotation, and attention with a
sliding window (ctypes binding of the same calls in include/gnn.h; argument marshalling only).

All tensors are views [rows, heads, head_dim] on the current device whose last stride is 1, so slices of a packed
projection are taken as they are."""
from __future__ import annotations

import ctypes
import math
import struct

from . import binding
from .binding import GNN_OK, GnnError

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


# The structures are packed into bytes that belong to one call: threads may call at once, each on its own stream.
_HEADS = struct.Struct("PqqiI").pack                         # GnnHeads
_CALL = struct.Struct("ii" + "PqqiI" * 4 + "PPPqqiiiiiifi").pack   # GnnAttentionCall
assert struct.calcsize("PqqiI") == ctypes.sizeof(GnnHeads)
assert struct.calcsize("ii" + "PqqiI" * 4 + "PPPqqiiiiiifi") == ctypes.sizeof(GnnAttentionCall)
_lib = _torch = _raw_stream = _current_device = None
DTYPES = {}


def _library():
    """The library, loaded once more so that its calls keep the interpreter lock: they only enqueue work, and giving the
    lock up and taking it again would cost more than they do."""
    global _lib, _torch, _raw_stream, _current_device
    if _lib is None:
        import torch
        binding.load_library()
        lib = ctypes.PyDLL(binding.LIB_PATH)
        i = ctypes.c_int
        lib.gnn_rotary_init.argtypes = [_vp, _vp]
        lib.gnn_rope.argtypes = [_vp, i, i, _vp, _vp, _vp, i, _i64, _vp]
        lib.gnn_qk_norm_rope.argtypes = [_vp, i, i, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, i, _vp, _i64, _i64,
                                         _vp]
        lib.gnn_attention_run.argtypes = [_vp, _vp, _vp]
        for f in (lib.gnn_rotary_init, lib.gnn_rope, lib.gnn_qk_norm_rope, lib.gnn_attention_run):
            f.restype = i
        waits = binding.load_library()                       # these wait for the device, without the lock
        waits.gnn_attention_create.argtypes = [ctypes.POINTER(_vp)]
        waits.gnn_attention_create.restype = i
        waits.gnn_attention_status.argtypes = [_vp, _vp]
        waits.gnn_attention_status.restype = i
        waits.gnn_attention_destroy.argtypes = [_vp]
        waits.gnn_attention_destroy.restype = None
        DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        _lib, _torch = lib, torch
    return _lib


def _stream(stream, device):
    return _raw_stream(device) if stream is None else stream.cuda_stream


def _empty_like(x, stream):
    """Like x, in memory of the call's stream: what another stream's held before may still be in use there."""
    if stream is None:
        return _torch.empty_like(x)
    with _torch.cuda.stream(stream):
        return _torch.empty_like(x)


def _fields(x, dtype, device, dim):
    """A view's fields; x: cuda tensor [rows, heads, dim], last stride 1, of the given type, device and head size."""
    shape, stride = x.shape, x.stride()
    assert len(shape) == 3 and (stride[2] == 1 or shape[2] == 1), "a tensor [rows, heads, dim], last stride 1"
    assert x.dtype == dtype and x.get_device() == device and shape[2] == dim, "types, devices or head sizes differ"
    return x.data_ptr(), stride[0], stride[1], shape[1], 0


def _heads(x, dtype, device, dim):
    """A view as a gnn_heads, whose address a call is given."""
    return _HEADS(*_fields(x, dtype, device, dim))


def _kind(x):
    """(type, its number, device, head size) of a cuda tensor."""
    device, dtype = x.get_device(), x.dtype
    assert device >= 0, "a cuda tensor"
    assert device == _current_device(), "the tensors' device is not the current one, where calls launch"
    assert dtype in DTYPES, f"type {dtype} is not taken"
    return dtype, DTYPES[dtype], device, x.shape[2]


def _vector(x, n, dtype, device):
    """A contiguous cuda vector's address, or None."""
    if x is None:
        return None
    assert x.get_device() == device and x.dtype == dtype and x.numel() == n and x.is_contiguous(), \
        f"a contiguous {dtype} cuda tensor of {n} is wanted"
    return x.data_ptr()


def _positions(pos, n, device):
    if pos is None:
        return None, 0
    real = pos.dtype == _torch.float32
    return _vector(pos, n, _torch.float32 if real else _torch.int32, device), int(real)


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
        self.address = ctypes.addressof(self.table)


def rope(rot: Rotary, x, positions=None, out=None, stream=None):
    """x [rows, heads, dim] rotated by positions (cuda int32 or float32 [rows]; None: row numbers).  out may be x."""
    dtype, number, device, dim = _kind(x)
    n = x.shape[0]
    if out is None:
        out = _empty_like(x, stream)
    assert out.shape == x.shape
    pos, real = _positions(positions, n, device)
    if n == 0:
        return out
    rc = _lib.gnn_rope(rot.address, number, dim, _heads(x, dtype, device, dim), _heads(out, dtype, device, dim), pos, real,
                       n, _stream(stream, device))
    if rc != GNN_OK:
        raise GnnError(rc, "gnn_rope")
    return out


def qk_norm_rope(rot: Rotary, q, k, positions=None, v=None, q_gain=None, k_gain=None, eps: float = 1e-6, q_out=None,
                 k_out=None, v_out=None, rows=None, stream=None):
    """(q_out, k_out, v_out): q and k normalised for each head and rotated, v copied.  With rows (cuda int64 [rows]),
    row r of k and v goes to row rows[r] of k_out and v_out, which are then given."""
    dtype, number, device, dim = _kind(q)
    n, k_shape = q.shape[0], k.shape
    assert k_shape[0] == n and (v is None or v.shape == k_shape), "rows or key heads differ"
    assert rows is None or (k_out is not None and (v is None or v_out is not None)), "rows need k_out and v_out"
    assert v is not None or v_out is None, "v_out without v"
    if q_out is None:
        q_out = _empty_like(q, stream)
    if k_out is None:
        k_out = _empty_like(k, stream)
    if v is not None and v_out is None:
        v_out = _empty_like(v, stream)
    m = k_out.shape[0]
    assert q_out.shape == q.shape and (rows is not None or m == n), "outputs of other sizes"
    assert v is None or v_out.shape[0] == m, "k_out and v_out differ"
    pos, real = _positions(positions, n, device)
    at = _vector(rows, n, _torch.int64, device)
    gq, gk = _vector(q_gain, dim, _torch.float32, device), _vector(k_gain, dim, _torch.float32, device)
    if n == 0:
        return q_out, k_out, v_out
    assert m > 0, "k_out has no rows"
    values, values_out = (None, None) if v is None else (_heads(v, dtype, device, dim), _heads(v_out, dtype, device, dim))
    rc = _lib.gnn_qk_norm_rope(rot.address, number, dim, eps, gq, gk, _heads(q, dtype, device, dim),
                               _heads(k, dtype, device, dim), values, _heads(q_out, dtype, device, dim),
                               _heads(k_out, dtype, device, dim), values_out, pos, real, at, m, n, _stream(stream, device))
    if rc != GNN_OK:
        raise GnnError(rc, "gnn_qk_norm_rope")
    return q_out, k_out, v_out


class WindowAttention:
    """One handle of gnn_attention_create on the current device (a stream's own; see include/gnn.h)."""

    def __init__(self):
        _library()
        h = _vp()
        rc = binding.load_library().gnn_attention_create(ctypes.byref(h))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_attention_create")
        self.handle, self.device = h, _current_device()

    def __call__(self, q, k, v, q_start, left: int = -1, right: int = -1, sinks: int = 0, scale=None, kv_start=None,
                 kv_len=None, max_q: int = 0, max_kv: int = 0, out=None, stream=None):
        """Attention of the queries q [rows, heads, dim] over the keys and values k, v [kv rows, kv heads, dim], bf16 or
        fp16.  q_start: cuda int32 [sequences + 1]; kv_start, kv_len: cuda int32 [sequences], or None: a sequence's keys
        are the rows of its queries.  left, right: keys visible before and after a query's own position (-1: all),
        sinks: first keys that stay visible; max_q, max_kv: the most queries and keys of a sequence, when known."""
        dtype, number, device, dim = _kind(q)
        assert device == self.device, "the handle belongs to another device"
        if out is None:
            out = _empty_like(q, stream)
        n, int32, rows = q_start.numel() - 1, _torch.int32, k.shape[0]
        assert n >= 0 and out.shape == q.shape and v.shape[0] == rows, "outputs, keys or values of other sizes"
        call = _CALL(number, dim, *_fields(q, dtype, device, dim), *_fields(k, dtype, device, dim),
                     *_fields(v, dtype, device, dim), *_fields(out, dtype, device, dim),
                     _vector(q_start, n + 1, int32, device), _vector(kv_start, n, int32, device) or 0,
                     _vector(kv_len, n, int32, device) or 0, q.shape[0], rows, n, max_q, max_kv, left, right, sinks,
                     1.0 / math.sqrt(dim) if scale is None else scale, 0)
        rc = _lib.gnn_attention_run(self.handle, call, _stream(stream, device))
        if rc != GNN_OK:
            raise GnnError(rc, "gnn_attention_run")
        return out

    def status(self, stream=None) -> int:
        return binding.load_library().gnn_attention_status(self.handle, binding._stream_handle(stream))

    def close(self):
        if getattr(self, "handle", None):
            binding.load_library().gnn_attention_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
