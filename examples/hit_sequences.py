"""Hits read as a sequence: an encoder layer over whole events, and a decoder that extends tracks hit by hit.

    python examples/hit_sequences.py [hits per event] [events]

The encoder puts the hits of every event of a batch in order of azimuth, normalises and rotates queries and keys
(qk_norm_rope) and lets every hit attend to a window of that order and to a few first tokens of its event, which stay
visible to all (WindowAttention; those tokens themselves see the window of their own places).  The decoder keeps keys and values of each track's hits in a cache: each step puts the new
hits' in their rows (the same call), attends with one query to a track, and drops the oldest hits by renumbering the
rest (rope, on the cached keys).  Weights are random: this shows how the calls fit together, not a trained model."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2402_09633_gb300 import InteractionNetwork, Rotary, WindowAttention, qk_norm_rope, rope  # noqa: E402
from paper_2402_09633_gb300 import synthetic as S  # noqa: E402


class HitLayer:
    """One attention layer: hidden = heads * dim wide, with kv key heads and gains for each head's elements."""

    def __init__(self, hidden=128, heads=2, kv=2, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv, self.dim, self.dtype = heads, kv, hidden // heads, dtype
        out = (heads + 2 * kv) * self.dim
        self.w_qkv = (torch.randn(hidden, out, generator=g, device="cuda") / math.sqrt(hidden)).to(dtype)
        self.w_out = (torch.randn(hidden, hidden, generator=g, device="cuda") / math.sqrt(hidden)).to(dtype)
        self.q_gain, self.k_gain = (1 + 0.1 * torch.randn(self.dim, generator=g, device="cuda") for _ in range(2))
        self.rotary = Rotary(self.dim)
        self.attend = WindowAttention()

    def project(self, h):
        qkv = (h @ self.w_qkv).view(h.shape[0], self.heads + 2 * self.kv, self.dim)
        return qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv], qkv[:, self.heads + self.kv:]

    def output(self, h, o):
        return h + o.reshape(h.shape) @ self.w_out

    def encode(self, h, starts, positions, left, right, sinks):
        """h [hits, hidden], the events' hits one after another from starts on, each event in its order."""
        q, k, v = self.project(h)
        q, k, v = qk_norm_rope(self.rotary, q, k, positions, v=v, q_gain=self.q_gain, k_gain=self.k_gain)
        return self.output(h, self.attend(q, k, v, starts, left=left, right=right, sinks=sinks))


class TrackCache:
    """Keys and values of the hits of `tracks` tracks, `capacity` rows each, and how many of them are there."""

    def __init__(self, layer, tracks, capacity):
        self.layer, self.capacity = layer, capacity
        self.k, self.v = (torch.zeros(tracks * capacity, layer.kv, layer.dim, dtype=layer.dtype, device="cuda")
                          for _ in range(2))
        self.first = torch.arange(tracks, device="cuda", dtype=torch.int32) * capacity
        self.length = torch.zeros(tracks, dtype=torch.int32, device="cuda")
        self.each = torch.arange(tracks + 1, device="cuda", dtype=torch.int32)

    def step(self, h, left, sinks):
        """One new hit of every track, h [tracks, hidden]: into the cache, and attended from."""
        layer = self.layer
        q, k, v = layer.project(h)
        q, _, _ = qk_norm_rope(layer.rotary, q, k, self.length, v=v, q_gain=layer.q_gain, k_gain=layer.k_gain, k_out=self.k,
                               v_out=self.v, rows=(self.first + self.length).long())
        self.length += 1
        return layer.output(h, layer.attend(q, self.k, self.v, self.each, left=left, right=0, sinks=sinks, kv_start=self.first,
                                            kv_len=self.length, max_q=1, max_kv=self.capacity))

    def drop(self, hits):
        """Forgets the first `hits` hits of every track (each has as many): the others move up, and their keys turn back by
        as many positions."""
        k, v = (x.view(-1, self.capacity, *x.shape[1:]) for x in (self.k, self.v))
        back = torch.full((k.shape[0] * (self.capacity - hits),), -hits, dtype=torch.int32, device="cuda")
        turned = rope(self.layer.rotary, k[:, hits:].reshape(-1, *self.k.shape[1:]), back)
        k[:, :self.capacity - hits] = turned.view_as(k[:, hits:])
        v[:, :self.capacity - hits] = v[:, hits:].clone()
        self.length -= hits


def event_batch(hits, events, net):
    """Embeddings [rows, hidden] of the hits of some events, each in order of azimuth behind its first tokens, the
    events' first rows and every row's position."""
    rows, starts = [], [0]
    for e in range(events):
        x, _ = S.generate_event(S.EventSpec(hits - e * (hits // 8), 0, "fanout"), e)
        x = torch.from_numpy(x[x[:, 1].argsort()]).cuda()
        rows.append(net.embed(x))
        starts.append(starts[-1] + GLOBALS + x.shape[0])
    width = rows[0].shape[1]
    g = torch.Generator(device="cuda").manual_seed(1)
    lift = torch.randn(width, 128, generator=g, device="cuda") / math.sqrt(width)
    tokens = torch.randn(GLOBALS, 128, generator=g, device="cuda")
    h = torch.cat([x for r in rows for x in (tokens, r @ lift)]).to(torch.bfloat16)
    positions = torch.cat([torch.arange(z - a, device="cuda", dtype=torch.int32) for a, z in zip(starts, starts[1:])])
    return h, torch.tensor(starts, dtype=torch.int32, device="cuda"), positions


GLOBALS = 16


def main(hits=30000, events=4):
    cfg = S.ModelConfig(3, 2, 64, 2, 2)
    net = InteractionNetwork(cfg, S.pack_blob(cfg, S.init_weights(cfg, 0)))
    net.load_embedding(S.pack_embed_blob(cfg, S.init_embed_weights(cfg)))
    h, starts, positions = event_batch(hits, events, net)
    layer = HitLayer()
    out = layer.encode(h, starts, positions, left=512, right=512, sinks=GLOBALS)
    assert layer.attend.status() == 0
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(10):
        layer.encode(h, starts, positions, left=512, right=512, sinks=GLOBALS)
    b.record()
    torch.cuda.synchronize()
    print(f"encoder layer: {events} events, {h.shape[0]} rows, window 512 + 512: {a.elapsed_time(b) / 10:.3f} ms")

    tracks, length = 1024, 12                                # tracks of hits next to each other in the order
    seeds = (torch.arange(tracks, device="cuda") * (h.shape[0] // tracks - length)).clamp(min=0)
    cache = TrackCache(layer, tracks, 16)
    for i in range(length):
        last = cache.step(out[seeds + i], left=7, sinks=2)
    cache.drop(4)
    last = cache.step(last, left=7, sinks=2)
    assert layer.attend.status() == 0 and bool(torch.isfinite(last).all())
    print(f"decoder: {tracks} tracks of {length} hits, four dropped, one more: {tuple(last.shape)}")


if __name__ == "__main__":
    main(*map(int, sys.argv[1:3]))
