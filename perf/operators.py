"""Attention over hits in order, and what stands around it, as cases that can be timed and compared.

Hits of an event put in order (of azimuth, or along a track) are read as a sequence: queries and keys are
normalised for each head and rotated by their positions, and each hit attends to a window of the order and to a
few first tokens that stay visible.  An encoder does that for all hits of an event, or of a batch of events, at
once; a decoder that extends tracks does it for one new hit of each track, over a cache of the earlier ones.

Each case names its operator in "op":
  rope    rope               the rotation alone, on [rows, heads, dim]
  norm    qk_norm_rope       norms of queries and keys, the rotation, and k and v put in their (cache) rows
  attend  WindowAttention    packed sequences, every row a query
  cached  WindowAttention    few new queries for each sequence, over a cache of `cap` rows for each
A window is (left, right) keys around a query's own position; -1: no bound.  `rows` counts queries over all
sequences.  Plain forms compute in 32 bits and round once.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _rope(name, **kw):
    c = {"name": name, "op": "rope", "type": "bf16", "rows": 1, "heads": 2, "dim": 64, "rot": 64, "layout": "half",
         "scaling": "none", "pos": "order"}
    c.update(kw)
    return c


def _norm(name, **kw):
    c = {"name": name, "op": "norm", "type": "bf16", "rows": 1, "heads": 2, "kv": 2, "dim": 64, "rot": 64, "layout": "half",
         "scaling": "none", "gains": True, "cap": 0}
    c.update(kw)
    return c


def _attend(name, **kw):
    c = {"name": name, "op": "attend", "type": "bf16", "rows": 1, "seqs": 1, "heads": 2, "kv": 2, "dim": 64, "left": 512,
         "right": 512, "sinks": 0}
    c.update(kw)
    return c


def _cached(name, **kw):
    c = {"name": name, "op": "cached", "type": "bf16", "rows": 1, "seqs": 1, "cap": 1, "heads": 16, "kv": 4, "dim": 128,
         "left": -1, "right": 0, "sinks": 0}
    c.update(kw)
    return c


def listed():
    return [
        # the smallest rotation: seven new hits, placed by their azimuth, fp32, part of the head
        _rope("rope_few_fp32", type="fp32", rows=7, heads=3, rot=20, layout="interleaved", pos="phi"),
        # every hit of a full event (300k hits, hidden width 128 as two heads), context scaled by parts
        _rope("rope_event", rows=300000, scaling="turns"),
        # one new token for each of 64 tracks, written into the cache
        _norm("norm_step", rows=64, heads=16, kv=4, dim=128, rot=128, cap=4096),
        # q, k, v of a full event out of one packed projection
        _norm("norm_event", rows=300000),
        # odd sizes: heads of 96, part of them rotated, shared keys, three ragged thousands of rows
        _norm("norm_odd_fp16", type="fp16", rows=10007, heads=6, kv=2, dim=96, rot=40, layout="interleaved", scaling="linear"),
        # the repository's tiny event as one sequence: latency counts
        _attend("attend_tiny", rows=2000, left=256, right=256, sinks=4),
        # a full event: 300k hits, 512 neighbours to each side, 16 global tokens
        _attend("attend_event", rows=300000, sinks=16),
        # seven ragged events, shared keys, heads of 96, looking back only, odd window
        _attend("attend_ragged_fp16", type="fp16", rows=30011, seqs=7, heads=6, kv=2, dim=96, left=1000, right=0, sinks=5),
        # one long causal sequence with a wide window: the most arithmetic
        _attend("attend_long", rows=16384, heads=8, kv=2, dim=128, left=4095, right=0, sinks=128),
        # one new token of one track: the smallest step
        _cached("cached_one", cap=4099, left=1023, sinks=4),
        # one new token for each of 64 sequences of up to 8192, nothing forgotten
        _cached("cached_batch", rows=64, seqs=64, cap=8192),
        # three new tokens each over eight long caches
        _cached("cached_long_fp16", type="fp16", rows=24, seqs=8, cap=131072, heads=8, kv=2),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges: any operator, sizes log-uniform, odd ones among them."""
    op = rng.choice(["rope", "norm", "attend", "attend", "cached", "cached"])
    dim = rng.choice([32, 64, 64, 96, 128, 128])
    kv = rng.choice([1, 2, 2, 4])
    heads = kv * rng.choice([1, 2, 3, 4])
    half = rng.choice(["bf16", "fp16"])
    if op in ("rope", "norm"):
        kind = rng.choice(["fp32", "bf16", "bf16", "fp16"])
        c = dict(type=kind, rows=_spread(rng, 1, 38e6 / (heads * dim * 2)), heads=heads, dim=dim,
                 rot=rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]),
                 layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "turns"]))
        if op == "rope":
            c = _rope(None, pos=rng.choice(["order", "phi"]), **c)
        else:
            c = _norm(None, kv=kv, gains=rng.random() < 0.8, cap=rng.choice([0, 1024]) if c["rows"] <= 256 else 0, **c)
    elif op == "attend":
        rows = _spread(rng, 100, 120000)
        left = _spread(rng, 16, max(17, min(4096, int(1.6e11 / (rows * heads * dim * 8)))))
        c = _attend(None, type=half, rows=rows, seqs=rng.choice([1, 1, 2, 5, 16]), heads=heads, kv=kv, dim=dim,
                    left=left, right=rng.choice([0, left, left // 3]), sinks=rng.choice([0, 1, 4, 16, 100]))
    else:
        seqs = _spread(rng, 1, 128)
        cap = _spread(rng, 16, min(131072, int(1.5e8 / (seqs * kv * dim))))
        c = _cached(None, type=half, seqs=seqs, rows=seqs * rng.choice([1, 1, 1, 2, 3]), cap=cap, heads=heads, kv=kv,
                    dim=dim, left=rng.choice([-1, -1, _spread(rng, 16, 4096)]), sinks=rng.choice([0, 4, 64]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------- shapes

def _lengths(case):
    """Queries and keys of every sequence: ragged, with the given sum (attend) or below the capacity (cached)."""
    n = case["seqs"]
    if case["op"] == "cached":
        f = (np.arange(1, n + 1) * 0.6180339887) % 1.0
        keys = np.maximum((case["cap"] * (0.5 + 0.5 * f)).astype(np.int64), 1) if n > 1 else np.array([case["cap"]])
        return np.full(n, case["rows"] // n, dtype=np.int64), keys
    f = 0.25 + (np.arange(1, n + 1) * 0.6180339887) % 1.0
    ends = np.round(np.cumsum(f) / f.sum() * case["rows"]).astype(np.int64)
    rows = np.diff(np.concatenate([[0], ends]))
    return rows, rows


def _frequencies(case):
    """Radians a position for each rotated pair, in 64 bits."""
    R = case["rot"]
    f = 10000.0 ** (-2.0 * np.arange(R // 2) / R)
    if case["scaling"] == "linear":
        f = f / 4.0
    elif case["scaling"] == "turns":
        g = np.clip((32768.0 * f / (2.0 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (g + (1.0 - g) / 8.0)
    return f


SCALINGS = {"none": None, "linear": ("linear", 4.0), "turns": ("turns", 8.0, 32768.0, 1.0, 32.0)}


def _visible(case):
    """Visible (query, key) pairs, and keys that some query sees, over all sequences."""
    left, right, sinks = case["left"], case["right"], case["sinks"]
    nq, nk = _lengths(case)
    pairs = keys = 0
    for n, L in zip(nq.tolist(), nk.tolist()):
        p = np.arange(L - n, L, dtype=np.int64)
        hi = np.clip(p + right if right >= 0 else np.full(n, L - 1), -1, L - 1)
        lo = np.clip(p - left if left >= 0 else np.zeros(n, np.int64), 0, None)
        first = np.minimum(np.minimum(sinks, lo), hi + 1)          # sinks before the window
        pairs += int((np.maximum(hi + 1 - lo, 0) + np.maximum(first, 0)).sum())
        if n:
            keys += int(max(hi.max() + 1 - max(lo.min(), 0), 0) + min(sinks, lo.min()))
    return pairs, keys


def work(case):
    s = 4 if case["type"] == "fp32" else 2
    T, H, D = case["rows"], case["heads"], case["dim"]
    if case["op"] == "rope":
        return {"bytes": 2 * T * H * D * s + 4 * T, "flops": 3 * T * H * case["rot"]}
    if case["op"] == "norm":
        return {"bytes": 2 * T * (H + 2 * case["kv"]) * D * s + 4 * T, "flops": T * (H + case["kv"]) * (4 * D + 3 * case["rot"])}
    pairs, keys = _visible(case)
    return {"bytes": 2 * T * H * D * s + 2 * keys * case["kv"] * D * s, "flops": 4 * D * H * pairs}


# ------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["type"]]
    T, H, D = case["rows"], case["heads"], case["dim"]

    def normal(*size, scale=1.0):
        return (torch.randn(*size, generator=g, device=DEV) * scale).to(t)

    st = {"case": case}
    if case["op"] in ("rope", "norm"):
        if case.get("pos") == "phi":                       # azimuth over pi, as in the hits' features, in 256ths of a turn
            st["pos"] = 128.0 * (2.0 * torch.rand(T, generator=g, device=DEV) - 1.0)
        elif T <= 256:                                     # new tokens: somewhere in their sequences
            st["pos"] = torch.randint(0, 100000, (T,), generator=g, device=DEV, dtype=torch.int32)
        else:                                              # hits of an event, in order
            st["pos"] = torch.arange(T, device=DEV, dtype=torch.int32)
        f = _frequencies(case) / (2.0 * math.pi)           # turns a position, in pieces of 12 bits for exact products
        parts = []
        for _ in range(2):
            e = 2.0 ** (np.floor(np.log2(f)) - 11)
            hi = np.floor(f / e) * e
            parts.append(hi)
            f = np.where(f - hi > 0, f - hi, 1e-30)
        parts.append(f)
        st["turns"] = [torch.from_numpy(p).to(DEV, torch.float32) for p in parts]
        if own:
            from paper_2402_09633_gb300 import Rotary
            st["rot"] = Rotary(case["rot"], base=10000.0, layout=case["layout"], scaling=SCALINGS[case["scaling"]])
    if case["op"] == "rope":
        st["x"] = normal(T, H, D)
    elif case["op"] == "norm":
        K = case["kv"]
        qkv = normal(T, H + 2 * K, D, scale=1.5)           # one projection's output: q, k and v are slices of it
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        st["gq"] = st["gk"] = None
        if case["gains"]:
            st["gq"], st["gk"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV) for _ in range(2))
        if case["cap"]:                                    # each row its own sequence's cache of `cap` rows
            st["rows"] = (torch.arange(T, device=DEV) * case["cap"]
                          + torch.randint(0, case["cap"], (T,), generator=g, device=DEV))
            st["kc"], st["vc"] = (torch.zeros(T * case["cap"], K, D, dtype=t, device=DEV) for _ in range(2))
    else:
        K = case["kv"]
        nq, nk = _lengths(case)
        st["nq"], st["nk"] = nq, nk
        st["q_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)).to(DEV)
        if case["op"] == "attend":
            qkv = normal(T, H + 2 * K, D)
            st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
            st["kv_start"], st["kv_len"] = st["q_start"][:-1].contiguous(), torch.from_numpy(nk.astype(np.int32)).to(DEV)
        else:
            st["q"] = normal(T, H, D)
            st["k"], st["v"] = (normal(case["seqs"] * case["cap"], K, D) for _ in range(2))
            st["kv_start"] = (torch.arange(case["seqs"], device=DEV) * case["cap"]).to(torch.int32)
            st["kv_len"] = torch.from_numpy(nk.astype(np.int32)).to(DEV)
        if own:
            from paper_2402_09633_gb300 import WindowAttention
            st["attn"] = WindowAttention()
    return st


# ------------------------------------------------------------------------------------- plain forms

def _cos_sin(st):
    """cos and sin [rows, 1, pairs] of position times frequency, reduced to less than a turn by exact products."""
    pos = st["pos"].float()[:, None]
    high = 4096.0 * torch.trunc(pos / 4096.0)
    mid = torch.trunc(pos - high)
    low = pos - high - mid
    a, b, c = st["turns"]
    t = sum(x - torch.round(x) for x in (high * a, mid * a, low * a, high * b, mid * b, low * b, pos * c))
    t = (t - torch.round(t)) * (2.0 * math.pi)
    return torch.cos(t)[:, None], torch.sin(t)[:, None]


def _rotate(case, x, cos, sin):
    R = case["rot"]
    r, rest = x[..., :R], x[..., R:]
    if case["layout"] == "half":
        u, w = r[..., :R // 2], r[..., R // 2:]
        return torch.cat([u * cos - w * sin, w * cos + u * sin, rest], -1)
    u, w = r[..., 0::2], r[..., 1::2]
    return torch.cat([torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2), rest], -1)


def _plain_norm(case, x, gain, cos, sin):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    return _rotate(case, x if gain is None else x * gain, cos, sin).to(TYPES[case["type"]])


def _plain_attention(st):
    """Query blocks of up to 128 rows, each with the keys of its window gathered, and the sinks before it."""
    case = st["case"]
    H, K, D, left, right, sinks = (case[n] for n in ("heads", "kv", "dim", "left", "right", "sinks"))
    G = H // K
    c = min(128, int(st["nq"].max()))
    blocks = -(-st["nq"] // c)
    seq = torch.from_numpy(np.repeat(np.arange(case["seqs"]), blocks)).to(DEV)
    at = torch.from_numpy(np.concatenate([np.arange(n) for n in blocks]) * c).to(DEV)
    nq = torch.diff(st["q_start"]).long()[seq]
    nk = st["kv_len"].long()[seq]
    i = at[:, None] + torch.arange(c, device=DEV)                              # [blocks, c] query in its sequence
    rows = (st["q_start"].long()[seq][:, None] + i).clamp(max=case["rows"] - 1)
    p = nk[:, None] - nq[:, None] + i                                          # its position among the keys
    longest = int(st["nk"].max())
    ahead = right if right >= 0 else longest
    if left < 0 or left + ahead + c + sinks >= longest:                        # all keys
        j = torch.arange(longest, device=DEV).expand(seq.numel(), longest)
        again = torch.zeros_like(j, dtype=torch.bool)
    else:                                                                      # the window, and the sinks before it
        j = p[:, :1] - left + torch.arange(c + left + ahead, device=DEV)
        j = torch.cat([torch.arange(sinks, device=DEV).expand(seq.numel(), sinks), j], 1)
        again = (torch.arange(j.shape[1], device=DEV) < sinks) & (j >= p[:, :1] - left)
    inside = (j >= 0) & (j < nk[:, None]) & ~again
    seen = inside[:, None, :] & torch.ones_like(p, dtype=torch.bool)[:, :, None]
    if right >= 0:
        seen &= j[:, None, :] <= p[:, :, None] + right
    if left >= 0:
        seen &= (j[:, None, :] >= p[:, :, None] - left) | (j[:, None, :] < sinks)
    at = (st["kv_start"].long()[seq][:, None] + torch.where(inside, j, 0)).clamp(max=st["k"].shape[0] - 1)
    k = st["k"][at].float().permute(0, 2, 3, 1)                                # [blocks, K, D, J]
    v = torch.where(inside[:, :, None, None], st["v"][at].float(), 0.0).permute(0, 2, 1, 3)
    q = st["q"][rows].float().view(seq.numel(), c, K, G, D).permute(0, 2, 3, 1, 4).reshape(seq.numel(), K, G * c, D)
    s = (q @ k) * (1.0 / math.sqrt(D))
    s = torch.where(seen[:, None, None], s.view(seq.numel(), K, G, c, -1), -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(-1, keepdim=True)
    o = (e.view(seq.numel(), K, G * c, -1) @ v).view(seq.numel(), K, G, c, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(seq.numel(), c, H, D)
    return o[i < nq[:, None]].to(TYPES[case["type"]])


def run(st):
    case = st["case"]
    if case["op"] == "rope":
        if own:
            from paper_2402_09633_gb300 import rope
            return rope(st["rot"], st["x"], st["pos"])
        cos, sin = _cos_sin(st)
        return _rotate(case, st["x"].float(), cos, sin).to(st["x"].dtype)
    if case["op"] == "norm":
        if own:
            from paper_2402_09633_gb300 import qk_norm_rope
            return qk_norm_rope(st["rot"], st["q"], st["k"], st["pos"], v=st["v"], q_gain=st["gq"], k_gain=st["gk"],
                                eps=1e-6, k_out=st.get("kc"), v_out=st.get("vc"), rows=st.get("rows"))
        cos, sin = _cos_sin(st)
        q, k = _plain_norm(case, st["q"], st["gq"], cos, sin), _plain_norm(case, st["k"], st["gk"], cos, sin)
        if not case["cap"]:
            return q, k, st["v"].contiguous()
        st["kc"][st["rows"]] = k
        st["vc"][st["rows"]] = st["v"]
        return q, st["kc"], st["vc"]
    if own:
        cached = {} if case["op"] == "attend" else {"kv_start": st["kv_start"], "kv_len": st["kv_len"], "max_kv": case["cap"]}
        return st["attn"](st["q"], st["k"], st["v"], st["q_start"], left=case["left"], right=case["right"],
                          sinks=case["sinks"], max_q=int(st["nq"].max()), **cached)
    return _plain_attention(st)


# ------------------------------------------------------------------------------------- 64 bits

def _angles64(case, st):
    a = st["pos"].double()[:, None, None] * torch.from_numpy(_frequencies(case)).to(DEV)
    return torch.polar(torch.ones_like(a), a)


def _rotate64(case, x, turn):
    R = case["rot"]
    x = x.clone()
    pick = (slice(0, R // 2), slice(R // 2, R)) if case["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    z = torch.complex(x[..., pick[0]].contiguous(), x[..., pick[1]].contiguous()) * turn
    x[..., pick[0]], x[..., pick[1]] = z.real, z.imag
    return x


def _attention64(case, st):
    """Sequence by sequence, a slice of queries at a time against the keys from the slice's first to its last."""
    D, G = case["dim"], case["heads"] // case["kv"]
    left, right, sinks = case["left"], case["right"], case["sinks"]
    out = torch.zeros(case["rows"], case["heads"], D, dtype=torch.float64, device=DEV)
    first, start = st["q_start"].tolist(), st["kv_start"].tolist()
    for b in range(case["seqs"]):
        n, L = int(st["nq"][b]), int(st["nk"][b])
        step = 1024
        for a in range(0, n, step):
            z = min(n, a + step)
            p0, p1 = L - n + a, L - n + z - 1
            hi = L if right < 0 else min(L, p1 + right + 1)
            lo = 0 if left < 0 else max(0, p0 - left)
            if hi <= 0:
                continue
            j = torch.cat([torch.arange(0, min(sinks, lo, hi)), torch.arange(lo, max(lo, hi))]).to(DEV)
            p = torch.arange(p0, p1 + 1, device=DEV)[:, None]
            hide = torch.zeros(z - a, j.numel(), dtype=torch.bool, device=DEV)
            if right >= 0:
                hide |= j > p + right
            if left >= 0:
                hide |= (j < p - left) & (j >= sinks)
            q = st["q"][first[b] + a:first[b] + z].double().transpose(0, 1)                # [heads, n, D]
            k = st["k"][start[b] + j].double().transpose(0, 1).repeat_interleave(G, 0)
            v = st["v"][start[b] + j].double().transpose(0, 1).repeat_interleave(G, 0)
            w = torch.softmax((q @ k.transpose(1, 2) / math.sqrt(D)).masked_fill(hide, -math.inf), -1)
            w = torch.where(hide.all(1)[:, None], 0.0, w)
            out[first[b] + a:first[b] + z] = (w @ v).transpose(0, 1)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return _rotate64(case, st["x"].double(), _angles64(case, st))
    if case["op"] == "norm":
        turn, done = _angles64(case, st), []
        for x, gain in ((st["q"].double(), st["gq"]), (st["k"].double(), st["gk"])):
            y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + 1e-6)
            done.append(_rotate64(case, y if gain is None else y * gain.double(), turn))
        if not case["cap"]:
            return done[0], done[1], st["v"].double()
        kc, vc = st["kc"].double(), st["vc"].double()
        kc[st["rows"]], vc[st["rows"]] = done[1], st["v"].double()
        return done[0], kc, vc
    if case["rows"] * case["heads"] * case["dim"] * (abs(case["left"]) + abs(case["right"]) + 1024) > 4e11 and case["op"] == "attend":
        return None
    return _attention64(case, st)
