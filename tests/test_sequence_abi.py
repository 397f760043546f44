"""What the sequence operators refuse, before any device work (no GPU)."""
import ctypes

import pytest

from paper_2402_09633_gb300 import GnnError, Rotary, binding
from paper_2402_09633_gb300 import sequence as Q


@pytest.fixture(scope="module")
def lib():
    return Q._library()


def _config(**kw):
    c = dict(rot_dim=64, layout=0, scaling=0, reserved=0, base=10000.0, factor=1.0, length=1.0, slow=0.0, fast=1.0,
             amplitude=1.0)
    c.update(kw)
    return Q.GnnRotaryConfig(**c)


@pytest.mark.parametrize("bad", [
    dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=258), dict(rot_dim=-2), dict(layout=2), dict(layout=-1),
    dict(scaling=3), dict(scaling=-1), dict(base=0.0), dict(base=float("nan")), dict(base=float("inf")),
    dict(amplitude=float("inf")), dict(scaling=1, factor=0.0), dict(scaling=1, factor=-2.0), dict(reserved=1),
    dict(scaling=2, length=0.0), dict(scaling=2, slow=1.0, fast=1.0), dict(scaling=2, slow=-1.0),
    dict(scaling=2, fast=float("inf")), dict(scaling=2, slow=float("nan"))])
def test_rotary_table_refusals(lib, bad):
    out = Q.GnnRotary()
    assert lib.gnn_rotary_init(ctypes.byref(_config()), ctypes.byref(out)) == 0
    assert lib.gnn_rotary_init(ctypes.byref(_config(**bad)), ctypes.byref(out)) == -1
    assert lib.gnn_rotary_init(None, ctypes.byref(out)) == -1
    assert lib.gnn_rotary_init(ctypes.byref(_config()), None) == -1


def test_rotary_table_holds_the_frequencies():
    import math
    t = Rotary(20, base=500.0, scaling=("turns", 4.0, 100.0, 0.5, 3.0)).table
    for i in range(10):
        f = 500.0 ** (-2.0 * i / 20)
        g = min(1.0, max(0.0, (100.0 * f / (2 * math.pi) - 0.5) / 2.5))
        f *= g + (1 - g) / 4.0
        assert abs(t.turn_hi[i] + t.turn_lo[i] - f / (2 * math.pi)) <= 2.0 ** -46 * f
    with pytest.raises(GnnError):
        Rotary(65)
    with pytest.raises(AssertionError):
        Rotary(64, layout="third")
    with pytest.raises(AssertionError):
        Rotary(64, scaling=("linear",))


BUF = ctypes.create_string_buffer(4096)
AT = (ctypes.addressof(BUF) + 63) // 64 * 64


def _view(**kw):
    v = dict(data=AT, row_stride=128, head_stride=64, n_heads=2, reserved=0)
    v.update(kw)
    return Q.GnnHeads(**v)


def _ref(x):
    return None if x is None else ctypes.byref(x)


@pytest.mark.parametrize("bad", [
    dict(rot=None), dict(rot=Q.GnnRotary()), dict(dtype=3), dict(dtype=-1), dict(dim=62), dict(dim=65), dict(dim=258),
    dict(x=None), dict(y=None), dict(x=_view(data=None)), dict(x=_view(n_heads=0)), dict(x=_view(n_heads=3)),
    dict(x=_view(row_stride=-1)), dict(y=_view(head_stride=-64)), dict(x=_view(data=AT + 1)), dict(n=-1),
    dict(n=2 ** 31 - 1), dict(pos=AT + 2), dict(x=_view(reserved=1)), dict(x=_view(row_stride=2 ** 60))])
def test_rope_refusals(lib, bad):
    a = dict(rot=Rotary(64).table, dtype=1, dim=64, x=_view(), y=_view(), pos=AT, n=4)
    a.update(bad)
    assert lib.gnn_rope(_ref(a["rot"]), a["dtype"], a["dim"], _ref(a["x"]), _ref(a["y"]), a["pos"], 0, a["n"], None) == -1


@pytest.mark.parametrize("bad", [
    dict(rot=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(gain=AT + 1), dict(q=None), dict(k=None),
    dict(v=None), dict(vo=None), dict(qo=None), dict(ko=None), dict(v=_view(n_heads=1)), dict(ko=_view(n_heads=1)),
    dict(v=_view(n_heads=1), vo=_view(n_heads=1)), dict(rows=AT + 4), dict(out_rows=-1), dict(n=-1), dict(dim=32)])
def test_norm_refusals(lib, bad):
    a = dict(rot=Rotary(64).table, dtype=1, dim=64, eps=1e-6, gain=AT, q=_view(), k=_view(), v=_view(), qo=_view(),
             ko=_view(), vo=_view(), rows=AT, out_rows=10, n=4)
    a.update(bad)
    assert lib.gnn_qk_norm_rope(_ref(a["rot"]), a["dtype"], a["dim"], a["eps"], a["gain"], a["gain"], _ref(a["q"]),
                                _ref(a["k"]), _ref(a["v"]), _ref(a["qo"]), _ref(a["ko"]), _ref(a["vo"]), AT, 0,
                                a["rows"], a["out_rows"], a["n"], None) == -1


@pytest.mark.parametrize("bad", [
    dict(dtype=0), dict(dtype=3), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(sinks=-1), dict(n_q_rows=-1), dict(n_kv_rows=2 ** 31 - 1), dict(n_seqs=-1),
    dict(max_q=-1), dict(max_kv=-1), dict(kv_start=None), dict(kv_len=None), dict(q_start=None), dict(q_start=AT + 2),
    dict(q=_view(data=AT + 8)), dict(k=_view(row_stride=4)), dict(v=_view(head_stride=12)), dict(out=_view(data=None)),
    dict(k=_view(n_heads=1)), dict(q=_view(n_heads=3), out=_view(n_heads=3)), dict(out=_view(n_heads=4)),
    dict(reserved=1)])
def test_attention_refusals(lib, bad):
    a = dict(dtype=1, head_dim=64, q=_view(), k=_view(), v=_view(), out=_view(), q_start=AT, kv_start=AT, kv_len=AT,
             n_q_rows=4, n_kv_rows=4, n_seqs=1, max_q=0, max_kv=0, left=-1, right=-1, sinks=0, scale=0.125, reserved=0)
    a.update(bad)
    handle = ctypes.cast(ctypes.create_string_buffer(4096), ctypes.c_void_p)   # zeroed: not looked at before the checks
    call = Q.GnnAttentionCall(**a)
    assert lib.gnn_attention_run(handle, ctypes.byref(call), None) == -1
    assert lib.gnn_attention_run(None, ctypes.byref(call), None) == -1
    assert lib.gnn_attention_run(handle, None, None) == -1


def test_null_handles(lib):
    assert lib.gnn_attention_create(None) == -1
    assert lib._name == binding.load_library()._name
    assert binding.load_library().gnn_attention_status(None, None) == -1
    binding.load_library().gnn_attention_destroy(None)
