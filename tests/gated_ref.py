"""Plain 64-bit forms of the gated layer's operators, on the CPU, with bounds of
what float32 arithmetic and one final rounding may differ from them by.

Bounds.  A float32 sum of n products is within (n + 4) 2^-24 sum |products|
whatever its order.  The activations come from e = exp(-|z|) and 1 / (1 + e):
z is rounded some four times (4 |z| 2^-24), the fast exponential is within
2 |z| 2^-24 beside that and the reciprocal within 2^-23, and some ten further
roundings follow: (32 + 8 |z|) 2^-24 of each term's magnitude bounds a and its
derivative.  Past |g| = 110, and where exp's result would be no normal number,
a term is taken as zero: it is below 110 * 2^-126 there.  An error m of g moves
act(g) by at most 1.13 m (the largest slope: gelu's)."""
import math

import torch

U32 = 2.0 ** -24
LOST = 110 * 2.0 ** -126
ACTS = ("relu", "sigmoid", "silu", "gelu")


def act(kind, g):
    """(act(g), act'(g), bounds of both) in 64 bits."""
    if kind == "relu":
        return g.clamp(min=0.0), (g > 0).double(), 0.0 * g, 0.0 * g
    k = 2.0 * math.sqrt(2.0 / math.pi) if kind == "gelu" else 1.0
    z, dz = (k * (g + 0.044715 * g ** 3), k * (1.0 + 0.134145 * g * g)) if kind == "gelu" else (g, torch.ones_like(g))
    s, far = torch.sigmoid(z), torch.sigmoid(-z)
    r = (32.0 + 8.0 * z.abs()) * U32
    if kind == "sigmoid":
        return s, s * far, r * s + LOST, r * s * far + LOST
    d = g * s * far * dz
    return g * s, s + d, r * (g * s).abs() + LOST, r * (s + d.abs()) + LOST


def _groups(off):
    return [(e, slice(a, b)) for e, (a, b) in enumerate(zip(off, off[1:])) if b > a]


def forward(x, w, off, kind):
    """{name: (value, bound)} of h and gu; rows of no expert NaN (not to be written)."""
    x, w = x.double(), w.double()
    E, _, K, C = w.shape
    gu = torch.full((x.shape[0], 2 * K), float("nan"), dtype=torch.float64)
    m = torch.zeros_like(gu)
    for e, r in _groups(off):
        f = w[e].reshape(2 * K, C)
        gu[r] = x[r] @ f.t()
        m[r] = (C + 4) * U32 * (x[r].abs() @ f.abs().t())
    g, u, mg, mu = gu[:, :K], gu[:, K:], m[:, :K], m[:, K:]
    a, _, ma, _ = act(kind, g)
    ma = ma + 1.13 * mg
    return {"gu": (gu, m), "h": (a * u, ma * u.abs() + a.abs() * mu + ma * mu + U32 * (a * u).abs())}


def backward(dy, w2, gu, off, kind):
    """{name: (value, bound)} of dgu and h."""
    dy, w2, gu = dy.double(), w2.double(), gu.double()
    E, C, K = w2.shape
    dh = torch.full((dy.shape[0], K), float("nan"), dtype=torch.float64)
    m = torch.zeros_like(dh)
    for e, r in _groups(off):
        dh[r] = dy[r] @ w2[e]
        m[r] = (C + 4) * U32 * (dy[r].abs() @ w2[e].abs())
    g, u = gu[:, :K], gu[:, K:]
    a, da, ma, mda = act(kind, g)
    ua, d = u.abs(), dh.abs()
    dg, du, h = dh * u * da, dh * a, a * u
    mdg = (m * da.abs() + (d + m) * mda) * ua + 3 * U32 * dg.abs()
    mdu = m * a.abs() + (d + m) * ma + 2 * U32 * du.abs()
    return {"dgu": (torch.cat((dg, du), 1), torch.cat((mdg, mdu), 1)), "h": (h, ma * ua + U32 * h.abs())}
