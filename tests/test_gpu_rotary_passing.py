"""Elements past rot_dim pass through the rotation as they are, whatever lies beside them."""
import pytest
import torch

from tests import sequence_ref as R
from tests.test_gpu_sequence import _rand

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SIZES = [(64, 32), (96, 40), (128, 64), (256, 128), (64, 20), (50, 6), (250, 30)]     # head, rotated
BITS = {F32: torch.int32, BF16: torch.int16, F16: torch.int16}


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", SIZES)
def test_rope_passes_any_value(dim, rot, layout, dtype):
    from paper_2402_09633_gb300 import Rotary, rope
    x = _rand(40, 3, dim, dtype=dtype, seed=dim)
    for i, odd in enumerate((float("inf"), float("-inf"), float("nan"), -0.0)):   # each place past rot in some head
        for e in range(rot, dim):
            x[(e + 7 * i) % 40, (e + i) % 3, e] = odd
    pos = torch.arange(40, dtype=torch.int32) * 31
    got = rope(Rotary(rot, layout=layout, amplitude=1.25), x.cuda(), pos.cuda()).cpu()
    assert torch.equal(got[..., rot:].contiguous().view(BITS[dtype]), x[..., rot:].contiguous().view(BITS[dtype]))
    want, size = R.rotate(x, pos, rot, layout, amplitude=1.25)
    R.check_rotated(got[..., :rot], want[..., :rot], size[..., :rot], normed=False)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", SIZES)
def test_an_infinite_element_past_the_rotation_norms_the_others_to_zero(dim, rot, layout, dtype):
    """The mean of the squares is infinite: the element itself is inf / inf, every other one is x / inf."""
    from paper_2402_09633_gb300 import Rotary, qk_norm_rope
    rows = dim - rot
    x = _rand(rows, 2, dim, dtype=dtype, seed=rot)
    x[torch.arange(rows), 1, torch.arange(rot, dim)] = float("inf")
    gain = (1 + _rand(dim, dtype=F32, seed=1, scale=0.3)).cuda()
    pos = torch.arange(rows, dtype=torch.int32)
    for got in qk_norm_rope(Rotary(rot, layout=layout), x.cuda(), x.cuda(), pos.cuda(), q_gain=gain, k_gain=gain)[:2]:
        want, size = R.rotate(R.norm(x, gain.cpu(), 1e-6), pos, rot, layout)
        own = torch.zeros_like(want, dtype=torch.bool)
        own[torch.arange(rows), 1, torch.arange(rot, dim)] = True
        got = got.cpu()
        assert torch.isnan(want[own]).all() and torch.isnan(got[own]).all()
        keep = ~own
        R.check_rotated(got[keep], want[keep], size[keep], normed=True)
