"""Plain 64-bit statements of the sequence operators, and how far a result in fewer bits may be from them."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # relative rounding error
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}                # of subnormal results


def frequencies(rot, base=10000.0, scaling=None):
    f = torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    if scaling and scaling[0] == "linear":
        f = f / scaling[1]
    elif scaling and scaling[0] == "turns":
        _, factor, length, slow, fast = scaling
        g = ((length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * (g + (1 - g) / factor)
    return f


def rotate(x, pos, rot, layout, base=10000.0, scaling=None, amplitude=1.0):
    """x [rows, heads, dim] in 64 bits, and the sum of the magnitudes of the two terms of every element."""
    x = x.double().clone()
    a = pos.double()[:, None, None] * frequencies(rot, base, scaling)
    c, s = torch.cos(a) * amplitude, torch.sin(a) * amplitude
    i = torch.arange(rot // 2)
    u, w = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    xu, xw = x[..., u], x[..., w]
    size = x.abs()
    x[..., u], x[..., w] = xu * c - xw * s, xw * c + xu * s
    size[..., u] = size[..., w] = (xu.abs() + xw.abs()) * abs(amplitude)
    return x, size


def norm(x, gain, eps):
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return y if gain is None else y * gain.double()


def check_rotated(got, want, size, normed):
    """An angle is off by at most 2^-21 (a handful of fp32 roundings of at most half a turn), cos and sin by 2^-23 more,
    products and sums by 2^-23; a norm adds the rounding of the mean of up to 256 squares, 2^-18 at most with sqrt
    and gain.  Then one rounding."""
    tol = (2.0 ** -20 + (2.0 ** -17 if normed else 0.0)) * size + UNIT[got.dtype] * want.abs() + TINY[got.dtype]
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), f"off by up to {float((err / tol).max()):.2f} of what roundings allow"


def visible(nq, nk, left, right, sinks):
    p = torch.arange(nk - nq, nk)[:, None]
    j = torch.arange(nk)[None, :]
    see = torch.ones(nq, nk, dtype=torch.bool)
    if right >= 0:
        see &= j <= p + right
    if left >= 0:
        see &= (j >= p - left) | (j < sinks)
    return see


def attention(q, k, v, see, scale):
    """One sequence: q [nq, heads, dim], k, v [nk, kv heads, dim] -> out, and the tolerance of a result that multiplies
    v by weights rounded to q's type."""
    nq, H, D = q.shape
    G = H // k.shape[1]
    unit = UNIT[q.dtype]
    q64 = q.double().transpose(0, 1)
    k64, v64 = (x.double().transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
    s = q64 @ k64.transpose(1, 2) * scale
    s = torch.where(see[None], s, -math.inf)
    m = s.amax(-1, keepdim=True) if s.shape[-1] else torch.full((H, nq, 1), -math.inf, dtype=torch.float64)
    e = torch.where(see[None], torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
    total = e.sum(-1, keepdim=True)
    w = torch.where(total != 0, e / total, 0.0)
    # only visible values count: where(see) before the product, so that 0 * NaN is not formed
    o = torch.zeros(H, nq, D, dtype=torch.float64)
    size = torch.zeros_like(o)
    if see.any():
        for i in range(nq):
            vis = see[i]
            o[:, i] = (w[:, i, vis, None] * v64[:, vis]).sum(1)
            size[:, i] = (w[:, i, vis, None] * v64[:, vis].abs()).sum(1)
    # scores: sums of D products in fp32, then a scale and an exponential of a few units more
    a = (q64.abs() @ k64.abs().transpose(1, 2)) * abs(scale)
    a = torch.where(see[None] & torch.isfinite(a), a, 0.0).amax(-1, keepdim=True) if a.shape[-1] else torch.zeros_like(m)
    ds = (D + 4) * 2.0 ** -23 * a + 2.0 ** -20
    top = torch.where(torch.isfinite(v64), v64.abs(), 0.0).amax() if v64.numel() else 0.0
    lost = (2.0 ** -24 * top * see.sum(1)[None, :, None].double()) if q.dtype == torch.float16 else 0.0
    tol = (unit + 2 * ds) * size + unit * o.abs() + TINY[q.dtype] + lost
    return o.transpose(0, 1), tol.transpose(0, 1)


def check_attention(got, q, k, v, q_start, kv_start, kv_len, left, right, sinks, scale):
    """got and the inputs on the CPU; every sequence against attention()."""
    for b in range(len(q_start) - 1):
        a, z = q_start[b], q_start[b + 1]
        ks, n = kv_start[b], kv_len[b]
        if z == a:
            continue
        want, tol = attention(q[a:z], k[ks:ks + n], v[ks:ks + n], visible(z - a, n, left, right, sinks), scale)
        g = got[a:z].double()
        fine = torch.isfinite(want)
        same = torch.where(torch.isnan(want), torch.isnan(g), g == want)
        assert bool(same[~fine].all()), f"sequence {b}: values that are not finite differ"
        err = (g - want).abs()[fine]
        assert bool((err <= tol[fine]).all()), \
            f"sequence {b}: off by up to {float((err / tol[fine]).max()):.2f} of what roundings allow"
