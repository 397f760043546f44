"""Plain 64-bit statements of the operators over caches in pages and over hypotheses."""
import math

import torch

from tests import sequence_ref as R


def rows_of(table, page, b, a, z):
    """Rows of positions a .. z - 1 of sequence b."""
    j = torch.arange(a, z)
    return table[b].long()[j // page] * page + j % page


def check_attention(got, q, k, v, table, kv_len, page, q_start, groups, shared, scale):
    """got and the inputs on the CPU; every sequence against a plain statement over its keys, one after another."""
    first, part = {}, {}
    for g in range(len(shared or [])):
        for b in range(groups[g], groups[g + 1]):
            first[b], part[b] = groups[g], shared[g]
    for b in range(len(q_start) - 1):
        a, z, n = q_start[b], q_start[b + 1], kv_len[b]
        if z == a:
            continue
        s = min(part.get(b, 0), n)
        at = torch.cat([rows_of(table, page, first.get(b, b), 0, s), rows_of(table, page, b, s, n)])
        want, tol = R.attention(q[a:z], k[at], v[at], R.visible(z - a, n, -1, 0, 0), scale)
        g = got[a:z].double()
        fine = torch.isfinite(want)
        same = torch.where(torch.isnan(want), torch.isnan(g), g == want)
        assert bool((same | fine).all()), f"sequence {b}: values that are not finite differ"
        err = (g - want).abs()[fine]
        assert bool((err <= tol[fine]).all()), \
            f"sequence {b}: off by up to {float((err / tol[fine]).max()):.2f} of what roundings allow"


def best(logits, scores, beams, n, ended=None, end=0):
    """(scores, parents, tokens) in 64 bits: [groups, n] each."""
    x = logits.double()
    rows, vocab = x.shape
    value = torch.log_softmax(x, 1) + scores.double()[:, None]
    value = torch.where(torch.isnan(value) | (x == -math.inf), -math.inf, value)
    out = []
    for g in range(rows // beams):
        found = []
        for b in range(beams):
            row = g * beams + b
            if ended is not None and bool(ended[row]):
                found.append((float(scores[row]), b, end))
                continue
            v = value[row]
            top = v.topk(min(n, vocab)).values[-1]               # ties at the least: all of them
            found += [(float(v[t]), b, int(t)) for t in torch.nonzero(v >= top).flatten()[:vocab]]
        found = [f for f in found if f[0] > -math.inf]
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        found = found[:n] + [(-math.inf, 0, -1)] * max(0, n - len(found))
        out.append(found)
    return (torch.tensor([[f[0] for f in g] for g in out], dtype=torch.float64),
            torch.tensor([[f[1] for f in g] for g in out]), torch.tensor([[f[2] for f in g] for g in out]))


def value_error(want, vocab):
    """How far a value may be off: each of the row's exponentials by 2^-22 and by the rounding of its argument, which weighs
    log2(vocab) units of 2^-24 at most on average; a thread's sum by as many units of 2^-24 as it has terms, vocab / 256
    at most and 64 in a strip's chunk; then one rounding."""
    lse = 2.0 ** -22 + 2.0 ** -24 * (2 * math.log2(vocab + 1) + vocab / 256 + 64)
    return lse + 2.0 ** -23 * want.abs()
