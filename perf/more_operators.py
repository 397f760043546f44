"""A decoder that extends tracks by several hypotheses at once, as cases that can be timed and compared.

Each event has a batch of hypotheses (beams), all of which start with the event's own tokens.  Keys and values lie in
pages; a step appends the new hits' keys and values, attends over the event's tokens (once for all its hypotheses) and
over each hypothesis' own hits, scores every candidate hit, keeps the best continuations and moves the states of the
hypotheses that they continue.

Each case names its operator in "op":
  append   PagedCache.append   the rotation (and norms) of new keys and queries, keys and values put in their pages
  attend   PagedCache.attend   `hyps` hypotheses of `events` events, `nq` new queries each, over up to `shared` tokens of
                               the event and up to `own` of the hypothesis (both ragged)
  select   beam_select         the best of `beams` x `vocab` continuations for each of `events` events
  reorder  beam_reorder        states of hypotheses, or their paged caches, moved to those that continue them
Plain forms compute in 32 bits (64 for angles and for values that decide an order) and round once.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _append(name, **kw):
    c = {"name": name, "op": "append", "type": "bf16", "seqs": 1, "rows": 1, "old": 0, "page": 64, "heads": 16, "kv": 4, "dim": 128,
         "rot": 128, "layout": "half", "norm": True}
    c.update(kw)
    return c


def _attend(name, **kw):
    c = {"name": name, "op": "attend", "type": "bf16", "events": 1, "hyps": 1, "nq": 1, "shared": 0, "own": 1, "page": 64,
         "heads": 16, "kv": 4, "dim": 128}
    c.update(kw)
    return c


def _select(name, **kw):
    c = {"name": name, "op": "select", "type": "bf16", "events": 1, "beams": 4, "best": 4, "vocab": 1000, "hidden": 0.0,
         "ended": 0.0}
    c.update(kw)
    return c


def _reorder(name, **kw):
    c = {"name": name, "op": "reorder", "type": "bf16", "events": 1, "beams": 4, "width": 64, "layers": 0, "page": 64, "old": 0,
         "kv": 4, "dim": 128}
    c.update(kw)
    return c


def listed():
    return [
        # a step: one new hit of each of 256 hypotheses, queries and keys normalised
        _append("append_step", seqs=256, rows=256, old=250),
        # seven events' own tokens at once, behind what the pages hold already; heads of 96, part of them rotated, no norms
        _append("append_events_fp16", type="fp16", seqs=7, rows=30011, old=37, page=16, heads=6, kv=2, dim=96, rot=40,
                layout="interleaved", norm=False),
        # the smallest step: four hypotheses of the repository's tiny event (2,000 hits, 128 wide as two heads)
        _attend("attend_tiny", events=1, hyps=4, shared=2000, own=12, page=16, heads=2, kv=2, dim=64),
        # 64 hypotheses of one event of 16,384 tokens
        _attend("attend_event", hyps=64, shared=16384, own=48),
        # eight ragged events, odd group of query heads, heads of 96, three new queries each
        _attend("attend_events_fp16", type="fp16", events=8, hyps=13, nq=3, shared=8001, own=300, page=32, heads=6, kv=2, dim=96),
        # the most arithmetic: 512 hypotheses over 65,536 tokens
        _attend("attend_long", hyps=512, shared=65536, own=100, page=128),
        # nothing shared: 64 sequences with caches of their own
        _attend("attend_apart", events=64, hyps=1, shared=0, own=8192, page=16),
        # the smallest choice: four beams, a thousand candidates
        _select("select_tiny", type="fp32"),
        # 64 events of eight beams, some of them ended, some candidates ruled out
        _select("select_batch", events=64, beams=8, best=8, vocab=32003, hidden=0.25, ended=0.1),
        # sixteen full events: every one of 300,000 hits may continue each of sixteen beams
        _select("select_event_fp32", type="fp32", events=16, beams=16, best=16, vocab=300000, hidden=0.5),
        # hidden states and histories of 512 hypotheses into another buffer
        _reorder("reorder_states", events=64, beams=8, width=16384),
        # paged caches of eight layers, in place: open pages of 64 rows, four key heads of 128
        _reorder("reorder_caches", events=64, beams=8, layers=8, old=500),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the same ranges: any operator, sizes log-uniform, odd ones among them."""
    op = rng.choice(["append", "attend", "attend", "attend", "select", "select", "reorder"])
    half = rng.choice(["bf16", "bf16", "fp16"])
    kv, dim, page = rng.choice([1, 2, 2, 4]), rng.choice([32, 64, 64, 96, 128, 128]), rng.choice([16, 32, 64, 128])
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    if op == "append":
        seqs = _spread(rng, 1, 512)
        rows = max(seqs, _spread(rng, seqs, 8e7 / (heads * dim * 4))) if rng.random() < 0.6 else seqs
        c = _append(None, type=rng.choice([half, half, "fp32"]), seqs=seqs, rows=rows, old=rng.choice([0, rng.randint(1, 300)]),
                    page=page, heads=heads, kv=kv, dim=dim, rot=rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]),
                    layout=rng.choice(["half", "interleaved"]), norm=rng.random() < 0.5)
    elif op == "attend":
        events = _spread(rng, 1, 16)
        hyps, nq = _spread(rng, 1, 512 / events), rng.choice([1, 1, 1, 2, 4])
        own_most = _spread(rng, 1, min(4096, max(2, 4e8 / (events * hyps * kv * dim * 4))))
        shared = _spread(rng, 1, min(65536, max(2, 1e11 / (events * hyps * nq * heads * dim * 4)), 4e8 / (events * kv * dim * 4)))
        c = _attend(None, type=half, events=events, hyps=hyps, nq=nq, shared=rng.choice([shared, shared, shared, 0]),
                    own=max(nq, own_most), page=page, heads=heads, kv=kv, dim=dim)
    elif op == "select":
        events, beams = _spread(rng, 1, 64), _spread(rng, 1, 32)
        c = _select(None, type=rng.choice([half, half, "fp32"]), events=events, beams=beams, best=rng.choice([beams, beams, _spread(rng, 1, 64)]),
                    vocab=_spread(rng, 10, min(300000, 4e7 / (events * beams))), hidden=rng.choice([0.0, 0.3]),
                    ended=rng.choice([0.0, 0.2]))
    else:
        events, beams, caches = _spread(rng, 1, 64), _spread(rng, 1, 32), rng.random() < 0.5
        c = _reorder(None, type=rng.choice([half, "fp32"]), events=events, beams=beams,
                     width=_spread(rng, 1, min(65536, 2e7 / (events * beams))), layers=rng.randint(1, 8) if caches else 0, page=page,
                     old=rng.randint(0, 500), kv=kv, dim=dim)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------- shapes

def _ragged(n, most):
    """n lengths of up to `most`, at least one."""
    if n == 1:
        return np.array([most], dtype=np.int64)
    f = (np.arange(1, n + 1) * 0.6180339887) % 1.0
    return np.maximum((most * (0.5 + 0.5 * f)).astype(np.int64), 1)


def _parts(n, total):
    """n ragged numbers of the given sum, each at least one."""
    f = 0.25 + (np.arange(1, n + 1) * 0.6180339887) % 1.0
    ends = np.round(np.cumsum(f) / f.sum() * (total - n)).astype(np.int64)
    return np.diff(np.concatenate([[0], ends])) + 1


def _lengths(case):
    """Queries, keys, event and shared keys of every sequence."""
    if case["op"] == "append":
        nq = _parts(case["seqs"], case["rows"])
        return nq, nq + np.arange(case["seqs"]) % (case["old"] + 1), None, None
    seqs = case["events"] * case["hyps"]
    event = np.repeat(np.arange(case["events"]), case["hyps"])
    shared = _ragged(case["events"], case["shared"]) if case["shared"] else np.zeros(case["events"], np.int64)
    nq = np.full(seqs, case["nq"], dtype=np.int64)
    return nq, shared[event] + np.maximum(_ragged(seqs, case["own"]), nq), event, shared


def _frequencies(case):
    return 10000.0 ** (-2.0 * np.arange(case["rot"] // 2) / case["rot"])


def work(case):
    s = 4 if case["type"] == "fp32" else 2
    if case["op"] == "append":
        T, H, K, D = case["rows"], case["heads"], case["kv"], case["dim"]
        return {"bytes": 2 * T * (H + 2 * K) * D * s + 8 * case["seqs"], "flops": T * (H + K) * (4 * D + 3 * case["rot"])}
    if case["op"] == "attend":
        nq, nk, event, shared = _lengths(case)
        H, K, D = case["heads"], case["kv"], case["dim"]
        keys = int(shared.sum() + (nk - shared[event]).sum())
        pairs = int((nq * nk - nq * (nq - 1) // 2).sum())
        return {"bytes": 2 * int(nq.sum()) * H * D * s + 2 * keys * K * D * s, "flops": 4 * D * H * pairs}
    if case["op"] == "select":
        n = case["events"] * case["beams"] * case["vocab"]
        return {"bytes": n * s * (1 - case["ended"]) + 12 * case["events"] * case["best"], "flops": 5 * n}
    n = case["events"] * case["beams"]
    if case["layers"]:
        moved, read = _moves(case)
        row = 2 * case["layers"] * (case["old"] % case["page"]) * case["kv"] * case["dim"] * s + 4 * (case["old"] // case["page"] + 1)
        return {"bytes": (moved + read) * row + 8 * n, "flops": 0}
    return {"bytes": 2 * n * (case["width"] * s + 4 * HISTORY) + 4 * n, "flops": 0}


HISTORY = 96                                               # ids of hits that a hypothesis remembers


def _parents(case):
    """Parents within each event.  In place (caches) a continued hypothesis keeps its slot and the others are given up for
    continuations of those, about half of them; else as they come, sorted by score."""
    rng = np.random.default_rng(case["events"] * 1000 + case["beams"])
    n, B = case["events"], case["beams"]
    at = rng.integers(0, B, (n, B))
    if case["layers"]:
        stay = rng.random((n, B)) < 0.5
        stay[:, 0] |= ~stay.any(1)
        order = np.argsort(~stay, axis=1, kind="stable")   # those that stay, first
        pick = np.take_along_axis(order, at % stay.sum(1)[:, None], 1)
        at = np.where(stay, np.arange(B), pick)
    return at.astype(np.int32)


def _moves(case):
    """Slots that get another's state, and different ones that are read for that."""
    at = _parents(case)
    gets = at != np.arange(case["beams"])
    return int(gets.sum()), sum(len(np.unique(row[g])) for row, g in zip(at, gets))


# ------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*size, scale=1.0):
        return (torch.randn(*size, generator=g, device=DEV) * scale).to(t)

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(DEV)

    def pages(n, width):                                   # every sequence's pages, anywhere
        return torch.randperm(n * width, generator=g, device=DEV).to(torch.int32).view(n, width)

    st = {"case": case}
    if case["op"] == "select":
        n = case["events"] * case["beams"]
        x = torch.randn(n, case["vocab"], generator=g, device=DEV) * 2.0
        if case["hidden"]:                                 # candidates that are ruled out
            x.masked_fill_(torch.rand(n, case["vocab"], generator=g, device=DEV) < case["hidden"], -math.inf)
        st["logits"] = x.to(t)
        st["scores"] = -20.0 * torch.rand(n, generator=g, device=DEV)
        st["ended"] = torch.rand(n, generator=g, device=DEV) < case["ended"] if case["ended"] else None
        return st
    if case["op"] == "reorder":
        n = case["events"] * case["beams"]
        st["parents"] = ints(_parents(case).reshape(-1))
        if not case["layers"]:
            st["states"] = [normal(n, case["width"]),
                            torch.randint(0, 300000, (n, HISTORY), generator=g, device=DEV, dtype=torch.int32)]
            st["out"] = [torch.empty_like(x) for x in st["states"]]
            return st
        width = case["old"] // case["page"] + 1
        st["table"], st["len"] = pages(n, width), torch.full((n,), case["old"], device=DEV, dtype=torch.int32)
        st["pools"] = [tuple(normal(n * width * case["page"], case["kv"], case["dim"]) for _ in range(2)) for _ in range(case["layers"])]
        if own:
            from paper_2402_09633_gb300 import PagedCache
            st["caches"] = [PagedCache(k, v, st["table"], st["len"], case["page"]) for k, v in st["pools"]]
        return st
    H, K, D = case["heads"], case["kv"], case["dim"]
    nq, nk, event, shared = _lengths(case)
    n, T = nq.size, int(nq.sum())
    st["nq"], st["nk"], st["event"], st["shared"] = nq, nk, event, shared
    st["q_start"], st["len"] = ints(np.concatenate([[0], np.cumsum(nq)])), ints(nk)
    width = -(-int(nk.max()) // case["page"])
    if case["op"] == "attend" and case["shared"]:          # pages of an event's tokens are those of all its hypotheses
        most = -(-int(shared.max()) // case["page"])
        mine = -(-int((nk - shared[event] + shared[event] % case["page"]).max()) // case["page"])
        table = torch.zeros(n, width, dtype=torch.int32, device=DEV)
        ids = torch.randperm(case["events"] * most + n * mine, generator=g, device=DEV).to(torch.int32)
        full = torch.from_numpy(shared // case["page"]).to(DEV)[torch.from_numpy(event).to(DEV)][:, None]
        at = torch.arange(width, device=DEV)[None]
        every = ids[:case["events"] * most].view(case["events"], most)[torch.from_numpy(event).to(DEV)]
        each = ids[case["events"] * most:].view(n, mine)
        table = torch.where(at < full, every.gather(1, at.clamp(max=most - 1).expand(n, width)),
                            each.gather(1, (at - full).clamp(0, mine - 1)))
        st["table"], count = table.contiguous(), ids.numel()
    else:
        st["table"], count = pages(n, width), n * width
    if case["op"] == "append":
        st["kc"], st["vc"] = (torch.zeros(count * case["page"], K, D, dtype=t, device=DEV) for _ in range(2))
        qkv = normal(T, H + 2 * K, D, scale=1.5)           # one projection's output: q, k and v are slices of it
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        st["gq"] = st["gk"] = None
        if case["norm"]:
            st["gq"], st["gk"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV) for _ in range(2))
        if own:
            from paper_2402_09633_gb300 import Rotary
            st["rot"] = Rotary(case["rot"], base=10000.0, layout=case["layout"])
    else:
        st["kc"], st["vc"] = (normal(count * case["page"], K, D) for _ in range(2))
        st["q"] = normal(T, H, D)
        if case["shared"]:
            st["groups"] = ints(np.arange(case["events"] + 1) * case["hyps"])
            st["shared_len"] = ints(shared)
            _fill_open_pages(st, case, event, shared)      # the page that the event's tokens end in is each hypothesis' own
    if own:
        from paper_2402_09633_gb300 import PagedCache
        st["cache"] = PagedCache(st["kc"], st["vc"], st["table"], st["len"], case["page"])
    return st


def _fill_open_pages(st, case, event, shared):
    """The event's last tokens, in the page of each of its hypotheses that goes on behind them."""
    page = case["page"]
    e = torch.from_numpy(event).to(DEV)
    part = torch.from_numpy(shared).to(DEV)[e]
    first = torch.arange(0, event.size, case["hyps"], device=DEV)[e]
    entry = torch.div(part, page, rounding_mode="floor").clamp(max=st["table"].shape[1] - 1)[:, None]
    to, frm = (st["table"][rows].gather(1, entry).long() * page + torch.arange(page, device=DEV)
               for rows in (torch.arange(event.size, device=DEV), first))
    there = torch.arange(page, device=DEV)[None] < (part % page)[:, None]
    for x in (st["kc"], st["vc"]):
        x[to[there]] = x[frm[there]]


# ------------------------------------------------------------------------------------- plain forms

def _rows(st):
    """Every query row's sequence and position."""
    nq = torch.diff(st["q_start"]).long()
    seq = torch.repeat_interleave(torch.arange(nq.numel(), device=DEV), nq, output_size=int(st["nq"].sum()))
    i = torch.arange(seq.numel(), device=DEV) - st["q_start"].long()[seq]
    return seq, st["len"].long()[seq] - nq[seq] + i


def _rotate(case, x, cos, sin):
    R = case["rot"]
    r, rest = x[..., :R], x[..., R:]
    if case["layout"] == "half":
        u, w = r[..., :R // 2], r[..., R // 2:]
        return torch.cat([u * cos - w * sin, w * cos + u * sin, rest], -1)
    u, w = r[..., 0::2], r[..., 1::2]
    return torch.cat([torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2), rest], -1)


def _plain_append(st):
    case = st["case"]
    seq, pos = _rows(st)
    a = pos.double()[:, None, None] * torch.from_numpy(_frequencies(case)).to(DEV)
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    done = []
    for x, gain in ((st["q"], st["gq"]), (st["k"], st["gk"])):
        x = x.float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
        done.append(_rotate(case, x, cos, sin).to(st["q"].dtype))
    page = case["page"]
    row = st["table"][seq, torch.div(pos, page, rounding_mode="floor")].long() * page + pos % page
    st["kc"][row] = done[1]
    st["vc"][row] = st["v"]
    return done[0], st["kc"], st["vc"]


def _plain_attend(st):
    """The event's keys for all its hypotheses at once, each hypothesis' own for itself, one softmax over both."""
    case = st["case"]
    page, H, K, D, nq = (case[n] for n in ("page", "heads", "kv", "dim", "nq"))
    E, P, G = case["events"], case["hyps"], H // K
    q = st["q"].float().view(E, P, nq, K, G, D).permute(0, 3, 1, 2, 4, 5)                # [E, K, P, nq, G, D]
    length = st["len"].long().view(E, P)
    table = st["table"].long()
    scale = 1.0 / math.sqrt(D)

    def gather(x, seq, pos):
        pos = pos.clamp(0, table.shape[1] * page - 1)
        return x[table[seq, torch.div(pos, page, rounding_mode="floor")] * page + pos % page].float()

    shared = st["shared_len"].long() if case["shared"] else torch.zeros(E, dtype=torch.long, device=DEV)
    n_own = int((st["nk"] - st["shared"][st["event"]]).max())
    j = shared[:, None, None] + torch.arange(n_own, device=DEV)                          # [E, 1, n_own]
    seq = torch.arange(E * P, device=DEV).view(E, P, 1)
    k, v = (gather(st[n], seq, j).permute(0, 3, 1, 4, 2) for n in ("kc", "vc"))          # [E, K, P, D, n_own]
    p = length[..., None] - nq + torch.arange(nq, device=DEV)                            # [E, P, nq]
    seen = (j[:, :, None] <= p[..., None])[:, None, :, :, None]                          # [E, 1, P, nq, 1, n_own]
    v = torch.where((j < length[..., None])[:, None, :, None], v, 0.0)
    s = (q.reshape(E, K, P, nq * G, D) @ k * scale).view(E, K, P, nq, G, n_own)
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    if case["shared"]:
        longest = int(st["shared"].max())
        i = torch.arange(longest, device=DEV)[None]
        ks, vs = (gather(st[n], (torch.arange(E, device=DEV) * P)[:, None], i).permute(0, 2, 3, 1) for n in ("kc", "vc"))
        there = (i < shared[:, None])[:, None, None]                                     # [E, 1, 1, longest]
        vs = torch.where(there, vs, 0.0)
        x = q.reshape(E, K, P * nq * G, D) @ ks * scale
        x = torch.where(there, x, -math.inf)
        m = torch.maximum(m, x.amax(-1).view(E, K, P, nq, G, 1))
        x = torch.exp(x - m.view(E, K, -1, 1))
    s = torch.exp(s - m)
    total = s.sum(-1, keepdim=True)
    o = (s.view(E, K, P, nq * G, n_own) @ v.transpose(3, 4)).view(E, K, P, nq, G, D)
    if case["shared"]:
        total = total + x.sum(-1).view(E, K, P, nq, G, 1)
        o = o + (x @ vs.transpose(2, 3)).view(E, K, P, nq, G, D)
    return (o / total).permute(0, 2, 3, 1, 4, 5).reshape(E * P * nq, H, D).to(st["q"].dtype)


def _plain_select(st):
    case = st["case"]
    E, B, V, n = (case[x] for x in ("events", "beams", "vocab", "best"))
    x = st["logits"].double()
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    value = st["scores"].double()[:, None] + (x - (m + torch.log(torch.exp(x - m).sum(1, keepdim=True))))
    value = torch.where(x == -math.inf, -math.inf, value)
    if st["ended"] is not None:
        alone = torch.where(torch.arange(V, device=DEV) == 0, st["scores"].double()[:, None], -math.inf)
        value = torch.where(st["ended"][:, None], alone, value)
    value = value.view(E, B * V)
    n_have = min(n, B * V)
    least = torch.topk(value, n_have, 1).values[:, -1:]                                  # of these, the lowest indices
    over = value > least
    spare = n_have - over.sum(1, keepdim=True)
    even = value == least
    take = over | (even & (torch.cumsum(even, 1, dtype=torch.int32) <= spare))
    at = torch.arange(B * V, device=DEV)
    at = torch.topk(torch.where(take, at, B * V), n_have, 1, largest=False).values.sort(1).values
    best, order = torch.sort(value.gather(1, at), dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    none = best == -math.inf
    scores, parents, tokens = best.float(), torch.where(none, 0, at // V), torch.where(none, -1, at % V)
    if n_have < n:
        more = (E, n - n_have)
        scores = torch.cat([scores, torch.full(more, -math.inf, device=DEV)], 1)
        parents = torch.cat([parents, torch.zeros(more, dtype=torch.long, device=DEV)], 1)
        tokens = torch.cat([tokens, torch.full(more, -1, dtype=torch.long, device=DEV)], 1)
    return scores.reshape(-1), parents.reshape(-1).int(), tokens.reshape(-1).int()


def _plain_reorder(st):
    case = st["case"]
    n, B = case["events"] * case["beams"], case["beams"]
    slot = torch.arange(n, device=DEV)
    frm = slot - slot % B + st["parents"].long()
    if not case["layers"]:
        for x, y in zip(st["states"], st["out"]):
            y.copy_(x[frm])
        return st["out"]
    page, full = case["page"], case["old"] // case["page"]
    to, src = (st["table"][s, full].long()[:, None] * page + torch.arange(case["old"] % page, device=DEV) for s in (slot, frm))
    for pools in st["pools"]:
        for x in pools:
            x[to] = x[src]
    st["table"][:, :full] = st["table"][frm, :full]
    return [st["table"], st["len"], *(x for pools in st["pools"] for x in pools)]


def run(st):
    case = st["case"]
    if case["op"] == "append":
        if own:
            q = st["cache"].append(st["rot"], st["q_start"], st["k"], st["v"], q=st["q"], q_gain=st["gq"], k_gain=st["gk"],
                                   eps=1e-6 if case["norm"] else None)
            return q, st["kc"], st["vc"]
        return _plain_append(st)
    if case["op"] == "attend":
        if own:
            return st["cache"].attend(st["q"], st["q_start"], groups=st.get("groups"), shared=st.get("shared_len"), max_q=case["nq"])
        return _plain_attend(st)
    if case["op"] == "select":
        if own:
            from paper_2402_09633_gb300 import beam_select
            return beam_select(st["logits"], st["scores"], case["beams"], best=case["best"], ended=st["ended"])
        return _plain_select(st)
    if own:
        from paper_2402_09633_gb300 import beam_reorder
        if not case["layers"]:
            return beam_reorder(st["parents"], case["beams"], st["states"], out=st["out"])
        beam_reorder(st["parents"], case["beams"], caches=st["caches"])
        return [st["table"], st["len"], *(x for pools in st["pools"] for x in pools)]
    return _plain_reorder(st)


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        return _append64(case, st)
    if case["op"] == "attend":
        return _attend64(case, st)
    if case["op"] == "select":
        return _select64(case, st)
    return _reorder64(case, st)


def _append64(case, st):
    turn = torch.from_numpy(_frequencies(case)).to(DEV)
    R, page = case["rot"], case["page"]
    pick = (slice(0, R // 2), slice(R // 2, R)) if case["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    out, kc, vc = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV), st["kc"].double(), st["vc"].double()
    first = np.concatenate([[0], np.cumsum(st["nq"])])
    for b in range(case["seqs"]):
        a, z = int(first[b]), int(first[b + 1])
        pos = torch.arange(int(st["nk"][b]) - (z - a), int(st["nk"][b]), device=DEV)
        angle = pos.double()[:, None, None] * turn
        z1 = torch.polar(torch.ones_like(angle), angle)
        new = []
        for x, gain in ((st["q"][a:z].double(), st["gq"]), (st["k"][a:z].double(), st["gk"])):
            if case["norm"]:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + 1e-6) * gain.double()
            y = x.clone()
            c = torch.complex(x[..., pick[0]].contiguous(), x[..., pick[1]].contiguous()) * z1
            y[..., pick[0]], y[..., pick[1]] = c.real, c.imag
            new.append(y)
        out[a:z] = new[0]
        row = st["table"][b].long()[pos // page] * page + pos % page
        kc[row], vc[row] = new[1], st["v"][a:z].double()
    return out, kc, vc


def _attend64(case, st):
    """Event by event and key head by key head: keys from the pages as they lie, the event's through its first hypothesis."""
    D, G, P, page, nq = case["dim"], case["heads"] // case["kv"], case["hyps"], case["page"], case["nq"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)

    def rows(b, a, z):
        p = torch.arange(a, z, device=DEV)
        return st["table"][b].long()[p // page] * page + p % page

    for e in range(case["events"]):
        s = int(st["shared"][e])
        common = rows(e * P, 0, s)
        for h in range(case["kv"]):
            ks, vs = st["kc"][common, h].double(), st["vc"][common, h].double()
            q = st["q"][e * P * nq:(e + 1) * P * nq, h * G:(h + 1) * G].double()         # [P nq, G, D]
            x = (q.reshape(-1, D) @ ks.T).view(P, nq, G, s) / math.sqrt(D)
            for i in range(P):
                b = e * P + i
                L = int(st["nk"][b])
                mine = rows(b, s, L)
                y = q[i * nq:(i + 1) * nq] @ st["kc"][mine, h].double().T / math.sqrt(D)  # [nq, G, own]
                last = torch.arange(L - nq, L, device=DEV)[:, None, None]
                y = y.masked_fill(torch.arange(s, L, device=DEV) > last, -math.inf)
                w = torch.softmax(torch.cat([x[i], y], -1), -1)
                out[b * nq:(b + 1) * nq, h * G:(h + 1) * G] = w[..., :s] @ vs + w[..., s:] @ st["vc"][mine, h].double()
    return out


def _select64(case, st):
    """Event by event: the largest value again and again, its first place each time."""
    B, V, n = case["beams"], case["vocab"], case["best"]
    scores = torch.full((case["events"], n), -math.inf, dtype=torch.float64, device=DEV)
    parents = torch.zeros(case["events"], n, dtype=torch.int32, device=DEV)
    tokens = torch.full((case["events"], n), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(B * V, device=DEV)
    for e in range(case["events"]):
        mine = slice(e * B, (e + 1) * B)
        value = torch.log_softmax(st["logits"][mine].double(), 1) + st["scores"][mine, None].double()
        value[torch.isnan(value)] = -math.inf
        if st["ended"] is not None:
            done = st["ended"][mine]
            value[done] = -math.inf
            value[done, 0] = st["scores"][mine][done].double()
        value = value.view(-1)
        for i in range(min(n, B * V)):
            top = value.max()
            first = torch.where(value == top, at, B * V).min()
            good = top > -math.inf
            scores[e, i] = top
            parents[e, i] = torch.where(good, torch.div(first, V, rounding_mode="floor"), 0)
            tokens[e, i] = torch.where(good, first % V, -1)
            value = torch.where(at == first, -math.inf, value)
    return scores.view(-1), parents.view(-1), tokens.view(-1)


def _reorder64(case, st):
    """Nothing is computed: slot by slot, what its parent's held before."""
    B, page, full, part = case["beams"], case["page"], case["old"] // case["page"], case["old"] % case["page"]
    at = st["parents"].tolist()
    if not case["layers"]:
        return [torch.stack([x[i - i % B + a] for i, a in enumerate(at)]) for x in st["states"]]
    table, before = st["table"].tolist(), st["table"].clone()
    for k, v in st["pools"]:
        for x in (k, v):
            held = x.clone()
            for i, a in enumerate(at):
                to, frm = (page * table[j][full] for j in (i, i - i % B + a))
                x[to:to + part] = held[frm:frm + part]
    for i, a in enumerate(at):
        st["table"][i, :full] = before[i - i % B + a, :full]
    return [st["table"], st["len"], *(x for pools in st["pools"] for x in pools)]
