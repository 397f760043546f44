"""Making an attention handle and asking for its status, beside work on other streams."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _busy(seconds):
    torch.cuda._sleep(int(seconds * 2e9))


def test_a_new_handle_is_ready_for_any_stream():
    """Nothing of its making is still to come on a stream that others do not wait for."""
    from paper_2402_09633_gb300 import WindowAttention
    WindowAttention()                                        # the library is loaded
    torch.cuda.synchronize()
    main = torch.cuda.default_stream()
    _busy(0.5)
    assert not main.query()
    att = WindowAttention()
    assert main.query()
    att.close()


def test_status_leaves_nothing_for_later():
    """The word is read and cleared in the caller's stream, where the next call comes after it."""
    from paper_2402_09633_gb300 import WindowAttention
    att, side = WindowAttention(), torch.cuda.Stream()
    x = torch.zeros(20, 1, 64, dtype=torch.bfloat16, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")     # noqa: E731
    start, first, many, few = i32([0, 1]), i32([0]), i32([21]), i32([20])
    out = torch.zeros_like(x)
    att(x, x, x, start, kv_start=first, kv_len=few, max_q=1, out=out)         # the kernel is loaded, which waits for all
    assert att.status() == 0
    torch.cuda.synchronize()
    main = torch.cuda.default_stream()
    _busy(1.0)
    with torch.cuda.stream(side):
        for _ in range(3):
            att(x, x, x, start, kv_start=first, kv_len=many, max_q=1, out=out)
            assert att.status() == -5
            assert att.status() == 0
            att(x, x, x, start, kv_start=first, kv_len=few, max_q=1, out=out)
            assert att.status() == 0
    assert not main.query()                                  # none of it waited for the other stream's work
    torch.cuda.synchronize()


def test_a_handle_of_another_device_is_refused():
    """By the library, before it looks at anything else of the handle: zeros behind the number of a second device."""
    import ctypes
    from paper_2402_09633_gb300 import WindowAttention
    from paper_2402_09633_gb300.binding import GnnError
    x = torch.zeros(20, 1, 64, dtype=torch.bfloat16, device="cuda")
    starts = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    att = WindowAttention()
    own, att.handle = att.handle, ctypes.cast((ctypes.c_int * 64)(1), ctypes.c_void_p)
    with pytest.raises(GnnError) as e:
        att(x, x, x, starts)
    assert e.value.code == -1
    att.handle = own
    att(x, x, x, starts)
    assert att.status() == 0
