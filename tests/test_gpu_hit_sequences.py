"""The example that runs the sequence operators together: an encoder over events, and a decoder over caches that must
say the same of a track's hits as the encoder says of them at once."""
import pytest
import torch

from examples import hit_sequences as H

pytestmark = pytest.mark.gpu

# Both sides round to bf16 (2^-8) after the projection, the norm, the weights, the attention and the output, and the
# projections of one row and of many may add up in another order: a handful of units of the largest output.
TOL = 8 * 2.0 ** -8


def _near(a, b):
    a, b = a.float(), b.float()
    assert float((a - b).abs().max()) <= TOL * float(b.abs().max())


@pytest.mark.parametrize("heads,kv", [(2, 2), (2, 1), (1, 1)])
def test_decoder_steps_equal_the_encoder(heads, kv):
    layer = H.HitLayer(heads=heads, kv=kv, seed=heads)
    tracks, n, left, sinks = 5, 21, 6, 2
    h = torch.randn(tracks * n, 128, generator=torch.Generator().manual_seed(0)).cuda().bfloat16()
    starts = torch.arange(tracks + 1, dtype=torch.int32, device="cuda") * n
    positions = torch.arange(n, dtype=torch.int32, device="cuda").repeat(tracks)
    want = layer.encode(h, starts, positions, left, 0, sinks).view(tracks, n, 128)
    cache = H.TrackCache(layer, tracks, n + 3)
    for i in range(n):
        _near(cache.step(h.view(tracks, n, 128)[:, i].contiguous(), left, sinks), want[:, i])
    assert layer.attend.status() == 0


def test_dropped_hits_are_as_if_they_had_not_been():
    layer = H.HitLayer(seed=3)
    tracks, n, drop = 4, 10, 3
    h = torch.randn(n + 1, tracks, 128, generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    whole, late = H.TrackCache(layer, tracks, 16), H.TrackCache(layer, tracks, 16)
    for i in range(n):
        whole.step(h[i], -1, 0)
        if i >= drop:
            late.step(h[i], -1, 0)
    whole.drop(drop)
    assert torch.equal(whole.length, late.length)
    _near(whole.step(h[n], -1, 0), late.step(h[n], -1, 0))


def test_example_runs():
    H.main(hits=1500, events=2)
