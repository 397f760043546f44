"""Sequence operators that make their outputs, called on another stream than the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("kind", ["rope", "norm", "attend"])
def test_outputs_do_not_take_what_the_current_stream_still_reads(kind):
    """Memory that the current stream has given back, but still has to read, is not an output on another stream."""
    from paper_2402_09633_gb300 import Rotary, WindowAttention, qk_norm_rope, rope
    rows = 5000
    x = torch.randn(rows, 4, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    rot, att, side = Rotary(64), WindowAttention(), torch.cuda.Stream()
    call = {"rope": lambda **s: [rope(rot, x, **s)],
            "norm": lambda **s: qk_norm_rope(rot, x, x, v=x, **s),
            "attend": lambda **s: [att(x, x, x, starts, left=20, right=0, **s)]}[kind]
    want = [y.clone() for y in call()]
    held = [torch.full_like(x, 3.0) for _ in range(3)]
    places = [h.data_ptr() for h in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(int(2e8))
    sums = [h.float().sum() for h in held]
    del held
    got = call(stream=side)
    assert not set(places) & {y.data_ptr() for y in got}
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert [float(s) for s in sums] == [3.0 * x.numel()] * 3
    assert att.status() == 0
