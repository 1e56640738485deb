"""Plain 64-bit forms of the expert-block operators, on the CPU, with bounds of
what float32 arithmetic and one final rounding may differ from them by.

Bounds.  A value rounded once to bf16 (8 bits of significand) is within 2^-8 of
itself, to float32 2^-24.  A float32 sum of n products is within
(n + 4) 2^-24 sum |products| whatever its order.  A row's statistics come from
sums at most about 64 additions deep (a thread's 16 values, the lanes, the
waves), and what is computed from them takes a few tens of further roundings:
256 * 2^-24 of the sum of the magnitudes that enter a value bounds it."""
import torch

U32 = 2.0 ** -24
U_OUT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ROW = 256 * U32


def check(got, ref, mag, what):
    """|got - ref| <= rounding of ref + mag, elementwise; got in its own type, ref and mag in 64 bits."""
    g = got.detach().cpu().double()
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    assert torch.isfinite(g).all(), what + ": not finite"
    tol = U_OUT[got.dtype] * ref.abs() + mag + 1e-37
    bad = (g - ref).abs() > tol
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError("%s: %d of %d off, first %s: got %r, want %r +- %r" % (
            what, int(bad.sum()), bad.numel(), i, float(g[i]), float(ref[i]), float(tol[i])))


def bits(live, total=None):
    """Packed bits (int32 words) of a boolean tensor in linear order."""
    b = live.flatten().to(torch.int64)
    b = torch.nn.functional.pad(b, (0, -b.numel() % 32)).view(-1, 32)
    w = (b << torch.arange(32)).sum(1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


# -------------------------------------------------------------------- experts

def expert_fwd(x, w, off, relu):
    """(Y, bound) of the experts' rows; other rows NaN (not to be written)."""
    x, w = x.double(), w.double()
    y = torch.full((x.shape[0], w.shape[1]), float("nan"), dtype=torch.float64)
    m = torch.zeros_like(y)
    for e in range(w.shape[0]):
        r = slice(off[e], off[e + 1])
        y[r] = x[r] @ w[e].t()
        m[r] = (x.shape[1] + 4) * U32 * (x[r].abs() @ w[e].abs().t())
    return (y.clamp(min=0) if relu else y), m


def expert_bwd_data(dy, w, off, live):
    dy, w = dy.double(), w.double()
    dx = torch.full((dy.shape[0], w.shape[2]), float("nan"), dtype=torch.float64)
    m = torch.zeros_like(dx)
    for e in range(w.shape[0]):
        r = slice(off[e], off[e + 1])
        dx[r] = dy[r] @ w[e]
        m[r] = (dy.shape[1] + 4) * U32 * (dy[r].abs() @ w[e].abs())
    if live is not None:
        dx, m = torch.where(live | dx.isnan(), dx, 0.0), torch.where(live, m, 0.0)
    return dx, m


def expert_bwd_weight(x, dy, off):
    x, dy = x.double(), dy.double()
    E = len(off) - 1
    dw = torch.zeros((E, dy.shape[1], x.shape[1]), dtype=torch.float64)
    m = torch.zeros_like(dw)
    for e in range(E):
        r = slice(off[e], off[e + 1])
        dw[e] = dy[r].t() @ x[r]
        m[e] = (off[e + 1] - off[e] + 4) * U32 * (dy[r].abs().t() @ x[r].abs())
    return dw, m


# ---------------------------------------------------------------------- norms

def _norm(v, kind, w, b, eps):
    """(N(v), n, mu, r, magnitude of n) in 64 bits."""
    if kind == "none":
        return v, v, None, None, v.abs()
    mu = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1.0 / ((v - mu).square().mean(1, keepdim=True) + eps).sqrt()
    n = (v - mu) * r
    size = n.abs() + (r * v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0)
    out = n
    if w is not None:
        out = out * w
    if b is not None:
        out = out + b
    return out, n, mu, r, size


def _d(t):
    return None if t is None else t.detach().cpu().double()


def _gates(gate, act, gate_rows, rows):
    if gate is None:
        return 1.0, 1.0, None
    g = gate[torch.arange(rows) // gate_rows]
    if act == "sigmoid":
        a = torch.sigmoid(g)
        # exp's argument is rounded: the relative error grows with |g|
        return a, a * (1 - a), 1.0 + g.abs() / 32
    return g, torch.ones_like(g), torch.ones_like(g)


def norm_fwd(x, u, gate, p, pre, post, act, gate_rows, eps):
    """{name: (value, bound)} of y, h and the statistics."""
    x, u, gate = _d(x), _d(u), _d(gate)
    p = {k: _d(v) for k, v in p.items()}
    out, my = {}, x.abs() * 0
    rows = x.shape[0]
    y, mu_u, r_u = x, None, None
    if u is not None:
        z, n, mu_u, r_u, size = _norm(u, post, p.get("w_post"), p.get("b_post"), eps)
        a, _, grow = _gates(gate, act, gate_rows, rows)
        s = 1.0 if p.get("scale") is None else p["scale"]
        y = x + s * a * z
        mz = size * (1.0 if p.get("w_post") is None else p["w_post"].abs()) + \
            (0.0 if p.get("b_post") is None else p["b_post"].abs())
        my = ROW * (x.abs() + abs(s * a) * mz * (1.0 if grow is None else grow))
        out["y"] = (y, my)
    if pre != "none":
        h, n, mu, r, size = _norm(y, pre, p.get("w_pre"), p.get("b_pre"), eps)
        w = 1.0 if p.get("w_pre") is None else p["w_pre"].abs()
        # y's own error, through the norm: its row's share and its own
        through = r * (my + my.mean(1, keepdim=True) * (1 + n.abs()))
        out["h"] = (h, ROW * (size * w + (0.0 if p.get("b_pre") is None else p["b_pre"].abs())) + through * w * 2)
        out["mu"], out["r"] = mu, r
    out["mu_u"], out["r_u"] = mu_u, r_u
    return out


def norm_bwd(y, u, gate, p, dy, dh, pre, post, act, gate_rows, eps):
    """{name: (value, bound)} of every gradient."""
    y, u, gate, dy, dh = _d(y), _d(u), _d(gate), _d(dy), _d(dh)
    p = {k: _d(v) for k, v in p.items()}
    rows = y.shape[0]
    one = lambda k: 1.0 if p.get(k) is None else p[k]  # noqa: E731
    summed = lambda v, m: (v.sum(0), (rows + 64) * U32 * v.abs().sum(0) + m.sum(0))  # noqa: E731
    out = {}

    def back(d, md, n, r, size, kind):
        c = d.mean(1, keepdim=True) if kind == "layer" else 0.0
        v = r * (d - c - n * (d * n).mean(1, keepdim=True))
        m = r * (md + md.mean(1, keepdim=True) + size * (md * size).mean(1, keepdim=True))
        return v, m

    gy = torch.zeros_like(y) if dy is None else dy
    mg = gy.abs()
    if pre != "none":
        _, n, _, r, size = _norm(y, pre, None, None, eps)
        out["w_pre"] = summed(dh * n, ROW * dh.abs() * size)
        out["b_pre"] = summed(dh, 0 * dh)
        v, m = back(dh * one("w_pre"), (dh * one("w_pre")).abs(), n, r, size, pre)
        gy, mg = gy + v, mg + m
    out["dx"] = (gy, ROW * mg)
    if u is None:
        return out
    _, n, _, r, size = _norm(u, post, None, None, eps)
    z = n * one("w_post") + (0.0 if p.get("b_post") is None else p["b_post"])
    mz = size * abs(one("w_post")) + (0.0 if p.get("b_post") is None else p["b_post"].abs())
    a, da, grow = _gates(gate, act, gate_rows, rows)
    grow = 1.0 if grow is None else grow
    s = one("scale")
    out["scale"] = summed(gy * a * z, ROW * mg * abs(a) * mz * grow)
    if gate is not None:
        dg = gy * s * z * da
        # 1 - a is rounded at 1: its error is not relative to a small derivative
        m = ROW * mg * abs(s) * mz * (abs(da) + (abs(a) * 2.0 ** -6 if act == "sigmoid" else 0)) * grow
        if gate_rows > 1:
            at = torch.arange(rows) // gate_rows
            zero = torch.zeros_like(gate)
            m = zero.index_add(0, at, m + (gate_rows + 64) * U32 * dg.abs())
            dg = zero.index_add(0, at, dg)
        out["dgate"] = (dg, m)
    dz, mdz = gy * s * a, mg * abs(s * a) * grow
    out["w_post"] = summed(dz * n, ROW * mdz * size)
    out["b_post"] = summed(dz, ROW * mdz)
    d, md = dz * one("w_post"), mdz * abs(one("w_post"))
    v, m = (d, md) if post == "none" else back(d, md, n, r, size, post)
    out["du"] = (v, ROW * m)
    return out
