"""What moving hypotheses' states refuses where arrays are given twice, before any device work (no GPU)."""
import ctypes

import pytest

from paper_2402_09633_gb300 import paged as G
from tests.test_paged_abi import AT, _pages, _view, lib  # noqa: F401


def test_one_array_of_two_states(lib):  # noqa: F811
    s = dict(data=AT, out=AT + 1024, stride=8, out_stride=8, row_bytes=8)
    for other in (dict(data=AT + 512), dict(), dict(stride=16)):
        both = (G.GnnBeamState * 2)(G.GnnBeamState(**s), G.GnnBeamState(**{**s, **other}))
        for groups in (0, 2):
            assert lib.gnn_beam_reorder(AT, groups, 3, both, 2, None) == -1
    nothing = (G.GnnBeamState * 3)(*[G.GnnBeamState(**{**s, "row_bytes": 0}) for _ in range(2)], G.GnnBeamState(**s))
    assert lib.gnn_beam_reorder(AT, 0, 3, nothing, 3, None) == 0


@pytest.mark.parametrize("other", [dict(k=_view(row_stride=256)), dict(v=_view(head_stride=128)), dict(dtype=0), dict(head_dim=32),
                                   dict(k=_view(n_heads=1), v=_view(n_heads=1))])
def test_one_pool_seen_as_two(lib, other):  # noqa: F811
    both = (G.GnnPages * 2)(_pages(n_seqs=0), _pages(n_seqs=0, **other))
    assert lib.gnn_paged_reorder(both, 2, AT, 0, 3, None) == -1
    same = (G.GnnPages * 3)(*[_pages(n_seqs=0)] * 3)
    assert lib.gnn_paged_reorder(same, 3, AT, 0, 3, None) == 0
