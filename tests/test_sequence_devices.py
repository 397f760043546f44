"""The sequence binding refuses tensors and handles of another device than the current one, where its calls would launch
(no GPU: a stand-in library and stand-in device numbers)."""
from contextlib import closing

import pytest

from paper_2402_09633_gb300 import sequence as Q
from tests.test_sequence_threads import Tensor, _calls, patched, stand_in   # noqa: F401


@pytest.mark.parametrize("kind,n", [("rope", 3), ("norm", 3), ("norm", 4), ("attend", 3)])
def test_tensors_of_another_device(patched, monkeypatch, kind, n):          # noqa: F811
    with closing(Q.WindowAttention()) as attend:
        call = _calls(kind, n, attend)
        call()
        monkeypatch.setattr(Q, "_current_device", lambda: 1)
        with pytest.raises(AssertionError):
            call()


def test_a_handle_of_another_device(patched, monkeypatch):                  # noqa: F811
    with closing(Q.WindowAttention()) as first:
        monkeypatch.setattr(Tensor, "device", 1)             # tensors and the current device move on
        with closing(Q.WindowAttention()) as second:
            with pytest.raises(AssertionError):
                _calls("attend", 3, first)()
            _calls("attend", 3, second)()
