"""What the operators over caches in pages and over hypotheses refuse, before any device work (no GPU)."""
import ctypes

import pytest

from paper_2402_09633_gb300 import Rotary, binding
from paper_2402_09633_gb300 import paged as G
from paper_2402_09633_gb300 import sequence as Q

BUF = ctypes.create_string_buffer(8192)
AT = (ctypes.addressof(BUF) + 63) // 64 * 64


@pytest.fixture(scope="module")
def lib():
    return G._library()


def _view(**kw):
    return Q.GnnHeads(**{**dict(data=AT, row_stride=128, head_stride=64, n_heads=2, reserved=0), **kw})


def _pages(**kw):
    return G.GnnPages(**{**dict(k=_view(), v=_view(), n_pages=4, dtype=1, head_dim=64, page_size=16, table_width=3, table=AT,
                                table_stride=3, kv_len=AT, n_seqs=2, reserved=0, status=AT), **kw})


BAD_PAGES = [dict(n_pages=0), dict(n_pages=2 ** 31), dict(n_pages=2 ** 26, page_size=64), dict(dtype=3), dict(dtype=-1),
             dict(head_dim=0), dict(head_dim=258), dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(page_size=0),
             dict(table_width=0), dict(table=None), dict(table=AT + 2), dict(kv_len=None), dict(kv_len=AT + 1), dict(table_stride=-1),
             dict(n_seqs=-1), dict(reserved=1), dict(k=_view(data=None)), dict(v=_view(n_heads=1)), dict(k=_view(row_stride=-1)),
             dict(v=_view(reserved=2)), dict(status=None), dict(status=AT + 2)]


@pytest.mark.parametrize("bad", [dict(pages=_pages(**b)) for b in BAD_PAGES] + [
    dict(pages=None), dict(rot=None), dict(rot=Q.GnnRotary()), dict(rot=Rotary(128).table), dict(call=None),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=0.0, q_gain=AT), dict(q_gain=AT + 2), dict(k_gain=AT + 1), dict(q_start=None),
    dict(q_start=AT + 2), dict(positions=AT + 1), dict(n_rows=-1), dict(n_rows=2 ** 31 - 1), dict(q=_view(data=None)),
    dict(q_out=_view(data=None)), dict(q_out=_view(n_heads=3)), dict(k=_view(n_heads=1)), dict(v=_view(data=None)),
    dict(k=_view(data=AT + 1)), dict(v=_view(head_stride=-1))])
def test_append_refusals(lib, bad):
    a = dict(pages=_pages(), rot=Rotary(64).table, call=1)
    c = dict(q=_view(), k=_view(), v=_view(), q_out=_view(), q_gain=None, k_gain=None, positions=AT, q_start=AT, n_rows=3, eps=1e-6,
             positions_float=0)
    for key, value in bad.items():
        (a if key in a else c)[key] = value
    ref = lambda x: None if x is None else ctypes.byref(x)   # noqa: E731
    call = a["call"] and G.GnnAppendCall(**c)
    assert lib.gnn_paged_append(ref(a["pages"]), ref(a["rot"]), ref(call), None) == -1


@pytest.mark.parametrize("bad", [dict(pages=_pages(**b)) for b in BAD_PAGES] + [
    dict(pages=None), dict(call=None), dict(pages=_pages(dtype=0)), dict(pages=_pages(head_dim=60)),
    dict(pages=_pages(head_dim=136)), dict(pages=_pages(k=_view(data=AT + 8))), dict(pages=_pages(v=_view(row_stride=4))),
    dict(pages=_pages(v=_view(row_stride=0))), dict(pages=_pages(k=_view(head_stride=0))), dict(scale=float("inf")),
    dict(scale=float("nan")), dict(n_q_rows=-1), dict(n_q_rows=2 ** 31 - 1), dict(max_q=-1), dict(n_groups=-1),
    dict(n_groups=2 ** 28 + 1), dict(n_groups=0), dict(group_start=None), dict(shared_len=None), dict(group_start=AT + 1),
    dict(shared_len=AT + 2), dict(q_start=None), dict(q_start=AT + 2), dict(q=_view(data=AT + 8)), dict(q=_view(row_stride=12)),
    dict(out=_view(data=None)), dict(out=_view(n_heads=4)), dict(q=_view(n_heads=3), out=_view(n_heads=3)),
    dict(q=_view(n_heads=4098), out=_view(n_heads=4098)), dict(q=_view(n_heads=258), out=_view(n_heads=258)), dict(reserved=1)])
def test_attend_refusals(lib, bad):
    a = dict(pages=_pages(), call=1)
    c = dict(q=_view(), out=_view(), q_start=AT, group_start=AT, shared_len=AT, n_q_rows=3, n_groups=1, max_q=0, scale=0.1, reserved=0,
             workspace=AT, workspace_bytes=2 ** 60)
    for key, value in bad.items():
        (a if key in a else c)[key] = value
    ref = lambda x: None if x is None else ctypes.byref(x)   # noqa: E731
    call, size = a["call"] and G.GnnPagedCall(**c), ctypes.c_uint64()
    assert lib.gnn_paged_attend(ref(a["pages"]), ref(call), None) == -1
    assert lib.gnn_paged_workspace(ref(a["pages"]), ref(call), ctypes.byref(size)) == -1
    assert lib.gnn_paged_workspace(ref(_pages()), ref(call), None) == -1


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(logits=AT + 1), dict(row_stride=-1), dict(n_groups=-1), dict(n_groups=2 ** 31 - 1), dict(scores=None),
    dict(scores=AT + 2), dict(dtype=3), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(best=0),
    dict(best=65), dict(reserved=1), dict(out_scores=None), dict(out_parents=AT + 1), dict(out_tokens=None), dict(workspace=None),
    dict(workspace=AT + 8), dict(workspace_bytes=0)])
def test_select_refusals(lib, bad):
    c = dict(logits=AT, row_stride=10, n_groups=2, scores=AT, ended=None, dtype=1, beams=3, vocab=10, best=3, end_token=0, reserved=0,
             out_scores=AT, out_parents=AT, out_tokens=AT, workspace=AT, workspace_bytes=2 ** 40)
    size = ctypes.c_uint64()
    assert lib.gnn_beam_workspace(ctypes.byref(G.GnnBeamCall(**c)), ctypes.byref(size)) == 0 and size.value > 0
    c.update(bad)
    assert lib.gnn_beam_select(ctypes.byref(G.GnnBeamCall(**c)), None) == -1
    assert lib.gnn_beam_select(None, None) == -1 and lib.gnn_beam_workspace(None, ctypes.byref(size)) == -1
    c["workspace_bytes"] = size.value - 1
    assert lib.gnn_beam_select(ctypes.byref(G.GnnBeamCall(**c)), None) == -1


@pytest.mark.parametrize("bad", [
    dict(parents=None), dict(parents=AT + 2), dict(n_groups=-1), dict(n_groups=2 ** 31 - 1), dict(beams=0), dict(beams=65),
    dict(n_states=-1), dict(states=None), dict(data=None), dict(out=None), dict(stride=7), dict(out_stride=7),
    dict(row_bytes=-1), dict(out=AT, out_stride=16)])
def test_reorder_refusals(lib, bad):
    a = dict(parents=AT, n_groups=2, beams=3, n_states=1, states=1)
    s = dict(data=AT, out=AT + 1024, stride=8, out_stride=8, row_bytes=8)
    for key, value in bad.items():
        (a if key in a else s)[key] = value
    states = a["states"] and ctypes.byref(G.GnnBeamState(**s))
    assert lib.gnn_beam_reorder(a["parents"], a["n_groups"], a["beams"], states, a["n_states"], None) == -1


@pytest.mark.parametrize("bad", [dict(pages=_pages(n_seqs=6, **b)) for b in BAD_PAGES if "n_seqs" not in b] + [
    dict(n_caches=0), dict(n_caches=-1), dict(pages=None), dict(parents=None), dict(parents=AT + 1), dict(beams=0),
    dict(beams=65), dict(n_groups=-1), dict(n_groups=3), dict(pages=_pages(n_seqs=5))])
def test_cache_reorder_refusals(lib, bad):
    a = dict(pages=_pages(n_seqs=6), n_caches=1, parents=AT, n_groups=2, beams=3)
    a.update(bad)
    ref = a["pages"] and ctypes.byref(a["pages"])
    assert lib.gnn_paged_reorder(ref, a["n_caches"], a["parents"], a["n_groups"], a["beams"], None) == -1


@pytest.mark.parametrize("other", [dict(table=AT + 64), dict(kv_len=AT + 64), dict(page_size=32), dict(table_stride=4), dict(n_pages=5),
                                   dict(table_width=2)])
def test_caches_that_are_reordered_together_have_one_table(lib, other):
    both = (G.GnnPages * 2)(_pages(n_seqs=6), _pages(n_seqs=6, **other))
    assert lib.gnn_paged_reorder(both, 2, AT, 2, 3, None) == -1


def test_status_words(lib):
    assert binding.load_library().gnn_paged_status(None, None) == -1
    assert binding.load_library().gnn_paged_status(AT + 1, None) == -1
