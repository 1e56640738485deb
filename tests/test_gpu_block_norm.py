"""Norms around a block with gate and residual scale, forward and backward,
against 64 bits."""
import pytest
import torch

import block_ref as ref
import paper_2109_07710_amd as cb

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
PARAMS = ("w_pre", "b_pre", "w_post", "b_post", "scale")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _strided(t, stride):
    if t is None:
        return None
    v = torch.full((t.shape[0], stride), float("nan"), dtype=t.dtype, device="cuda")[:, :t.shape[1]]
    v.copy_(t)
    return v


def _draw(rows, C, pre, post, gate, gate_rows, dtype, res, bias, scale, block, seed, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *n: torch.randn(n, generator=g)  # noqa: E731
    t = dict(x=(2 * rand(rows, C) + shift).to(DT[res]), u=None, gate=None, dy=rand(rows, C).to(DT[res]),
             dh=rand(rows, C).to(DT[dtype]) if pre != "none" else None)
    if block:
        t["u"] = (rand(rows, C) * 0.7 + 0.1 + shift).to(DT[dtype])
        if gate != "none":
            t["gate"] = (2 * rand(-(-rows // gate_rows), C)).to(DT[dtype])
    p = dict.fromkeys(PARAMS)
    if pre != "none":
        p["w_pre"] = 1 + 0.2 * rand(C)
        p["b_pre"] = 0.1 * rand(C) if bias else None
    if block and post != "none":
        p["w_post"] = 1 + 0.2 * rand(C)
        p["b_post"] = 0.1 * rand(C) if bias else None
    if block and scale:
        p["scale"] = 0.5 + 0.1 * rand(C)
    return t, p


def _run(rows, C, pre="rms", post="rms", gate="sigmoid", gate_rows=1, dtype="bf16", res="bf16", bias=False, scale=False,
         block=True, pad=0, seed=1, shift=0.0, dy=True):
    print("[case]", rows, C, pre, post, gate, gate_rows, dtype, res, flush=True)
    t, p = _draw(rows, C, pre, post, gate, gate_rows, dtype, res, bias, scale, block, seed, shift)
    s = [C + pad, C + 2 * pad, C + 3 * pad]
    d = cb.NormDesc.make(rows, C, pre, post, gate, gate_rows, dtype, res, EPS, *s)
    P = {k: None if v is None else v.cuda() for k, v in p.items()}
    params = cb.NormParams(*(P[k] for k in PARAMS))
    x, u, g = _strided(t["x"], s[0]), _strided(t["u"], s[1]), _strided(t["gate"], s[2])
    like = lambda v, st: None if v is None else _strided(torch.full_like(v, float("nan")), st)  # noqa: E731
    y = like(t["x"], s[0]) if block else None
    h = like(t["dh"], s[1])
    stats = torch.full((rows, 4), float("nan"), device="cuda")
    cb.block_norm_fwd(d, x, u, g, params, y, h, stats)
    want = ref.norm_fwd(t["x"], t["u"], t["gate"], p, pre, post, gate, gate_rows, EPS)
    if block:
        ref.check(y, *want["y"], "y")
    if pre != "none":
        ref.check(h, *want["h"], "h")
        assert torch.allclose(stats[:, 1].cpu().double(), want["r"][:, 0], rtol=2e-4 if block else 64 * ref.U32, atol=0)
    # backward from what the forward stored: the statistics of the stored
    # stream, so that the formula and the kernel start from the same numbers
    ys = (y if block else x).detach().cpu()
    st = torch.zeros((rows, 4), dtype=torch.float64)
    for k, v, kind in ((0, ys, pre), (2, t["u"], post)):
        if v is None or kind == "none":
            continue
        v = v.double()
        mu = v.mean(1) if kind == "layer" else torch.zeros(rows, dtype=torch.float64)
        st[:, k], st[:, k + 1] = mu, 1 / ((v - mu[:, None]).square().mean(1) + EPS).sqrt()
    stats = st.float().cuda()
    grads = {k: None if v is None else torch.full((C,), float("nan"), device="cuda") for k, v in p.items()}
    dx, du, dg = like(t["x"], s[0]), like(t["u"], s[1]), like(t["gate"], s[2])
    ws = cb.norm_workspace(d)
    ws.fill_(255)
    args = (d, _strided(ys, s[0]), u, g, params, stats, _strided(t["dy"], s[0]) if dy else None, _strided(t["dh"], s[1]))
    cb.block_norm_bwd(*args, dx, du, dg, cb.NormParams(*(grads[k] for k in PARAMS)), ws)
    want = ref.norm_bwd(ys, t["u"], t["gate"], p, t["dy"] if dy else None, t["dh"], pre, post, gate, gate_rows, EPS)
    for name, got in (("dx", dx), ("du", du), ("dgate", dg), *grads.items()):
        if got is not None:
            ref.check(got, *want[name], name)
    # again, and without the gradients nobody asks for: the same bits
    dx2, du2 = like(t["x"], s[0]), like(t["u"], s[1])
    w2 = None if grads["w_pre"] is None else torch.empty_like(grads["w_pre"])
    cb.block_norm_bwd(*args, dx2, du2, None, cb.NormParams(w2), ws)
    assert torch.equal(dx, dx2) and (du is None or torch.equal(du, du2)) and (w2 is None or torch.equal(w2, grads["w_pre"]))


# every way a row is laid over threads: part of a wave, a wave, several
SIZES = [(1, 8), (3, 64), (5, 72), (300, 8), (257, 200), (33, 512), (70, 520), (9, 1024), (2, 1032), (21, 2048), (5, 4104),
         (3, 8192), (2, 16384)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")], ids="-".join)
def test_sizes(size, types):
    _run(*size, dtype=types[0], res=types[1])
    _run(*size, "layer", "layer", "linear", 1, *types, bias=True, scale=True, pad=8)


@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "linear", "sigmoid"])
def test_forms(pre, post, gate):
    _run(37, 136, pre, post, gate, scale=True, bias=True)
    _run(37, 2056, pre, post, gate, dtype="bf16", res="f32")


@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_input_norm_alone(pre):
    """The first block's: h = N(x), no block before; dx with and without a dy."""
    _run(50, 264, pre, block=False, bias=True)
    _run(50, 264, pre, block=False, dy=False)
    _run(4, 5000, pre, block=False, dtype="f32", res="f32")


@pytest.mark.parametrize("rows,gate_rows,C", [(12, 3, 64), (100, 7, 72), (5, 5, 4096), (6, 100, 264), (3000, 1500, 64),
                                              (3000, 1499, 2048), (1030, 2, 128), (700, 300, 1032)])
def test_shared_gates(rows, gate_rows, C):
    """A gate row for several rows: groups shorter and longer than a
    workgroup's rows, a last one that is short, one group for all."""
    _run(rows, C, gate_rows=gate_rows)
    _run(rows, C, "layer", "layer", "linear", gate_rows, "f32", "f32", bias=True, scale=True, pad=16)


def test_far_from_zero():
    """Rows whose mean is a hundred deviations away: the squares are taken
    about the mean."""
    _run(20, 1000, "layer", "layer", "none", dtype="f32", res="f32", shift=100.0)
    _run(20, 3000, "layer", "layer", "none", dtype="f32", res="f32", shift=100.0)


def test_zero_rows_and_extremes():
    """Rows of zeros (r = 1 / sqrt(eps)), gates far out, and values whose
    squares still fit."""
    d = cb.NormDesc.make(4, 64, "layer", "rms", "sigmoid", eps=EPS)
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    u = torch.zeros_like(x)
    u[1] = 1e15
    u[2] = torch.linspace(-3, 3, 64)
    g = torch.full_like(x, 200.0)
    g[2, ::2], g[3] = -200.0, 0.0
    y, h, st = torch.empty_like(x), torch.empty_like(x), torch.empty((4, 4), device="cuda")
    cb.block_norm_fwd(d, x, u, g, None, y, h, st)
    assert (y[0] == 0).all() and (h[0] == 0).all() and (y[3] == 0).all()
    # (a row of equal values: its mean is rounded, and r = 1 / sqrt(eps) enlarges that)
    assert (y[1] == 1).all() and (h[1].float().abs() <= 64 * ref.U32 * EPS ** -0.5).all()
    assert (y[2, ::2] == 0).all() and torch.isfinite(h).all()
    assert torch.allclose(st[0, 1].cpu(), torch.tensor(EPS ** -0.5), rtol=1e-6)
    # a NaN stays in its row
    x[2, 3] = float("nan")
    cb.block_norm_fwd(d, x, u, g, None, y, h, st)
    assert torch.isnan(h[2]).all() and torch.isfinite(h[[0, 1, 3]]).all()


def test_in_place():
    """y over x and dx over dy: a program that keeps one stream buffer."""
    t, p = _draw(65, 520, "rms", "rms", "sigmoid", 1, "bf16", "bf16", False, False, True, 7)
    d = cb.NormDesc.make(65, 520, gate="sigmoid", eps=EPS)
    params = cb.NormParams(*(None if p[k] is None else p[k].cuda() for k in PARAMS))
    x, u, g = t["x"].cuda(), t["u"].cuda(), t["gate"].cuda()
    y, h, h2, st = torch.empty_like(x), torch.empty_like(u), torch.empty_like(u), torch.empty((65, 4), device="cuda")
    cb.block_norm_fwd(d, x, u, g, params, y, h, st)
    cb.block_norm_fwd(d, x, u, g, params, x, h2, st)
    assert torch.equal(x, y) and torch.equal(h, h2)
    dy, dh, ws = t["dy"].cuda(), t["dh"].cuda(), cb.norm_workspace(d)
    dx = torch.empty_like(dy)
    cb.block_norm_bwd(d, y, u, g, params, st, dy, dh, dx, None, None, None, ws)
    cb.block_norm_bwd(d, y, u, g, params, st, dy, dh, dy, None, None, None, ws)
    assert torch.equal(dx, dy)


@pytest.mark.parametrize("post,gate,gate_rows", [("layer", "sigmoid", 1), ("rms", "linear", 5), ("none", "sigmoid", 1)])
def test_gradients_are_differences(post, gate, gate_rows):
    """float32: along each gradient, L = sum(y dy) + sum(h dh) changes by its
    norm.  Step 2^-7 of a direction of norm 1 spread over the tensor: the
    cubic term is below 1e-4 of the slope, the sums' rounding (2^-24 of |L|'s
    terms, some hundreds, over the step) below 1e-2 of the smallest slope."""
    rows, C = 20, 136
    t, p = _draw(rows, C, "layer", post, gate, gate_rows, "f32", "f32", True, True, True, 8)
    d = cb.NormDesc.make(rows, C, "layer", post, gate, gate_rows, "f32", "f32", EPS)
    v = {k: t[k].cuda() for k in ("x", "u", "gate")}
    v.update({k: a.cuda() for k, a in p.items() if a is not None})
    dy, dh = t["dy"].cuda(), t["dh"].cuda()
    y, h, st = torch.empty_like(v["x"]), torch.empty_like(v["u"]), torch.empty((rows, 4), device="cuda")

    def loss(**change):
        a = {**v, **change}
        cb.block_norm_fwd(d, a["x"], a["u"], a["gate"], cb.NormParams(*(a.get(k) for k in PARAMS)), y, h, st)
        return float((y.double() * dy).sum() + (h.double() * dh).sum())

    loss()
    grads = {k: torch.empty_like(v[k]) for k in PARAMS if k in v}
    dx, du, dg = torch.empty_like(v["x"]), torch.empty_like(v["u"]), torch.empty_like(v["gate"])
    cb.block_norm_bwd(d, y.clone(), v["u"], v["gate"], cb.NormParams(*(v.get(k) for k in PARAMS)), st.clone(), dy, dh, dx, du,
                      dg, cb.NormParams(*(grads.get(k) for k in PARAMS)), cb.norm_workspace(d))
    for name, grad in (("x", dx), ("u", du), ("gate", dg), *grads.items()):
        n = float(grad.norm())
        step = grad / n * 2.0 ** -7
        slope = (loss(**{name: v[name] + step}) - loss(**{name: v[name] - step})) / 2.0 ** -6
        assert abs(slope - n) <= 1e-2 * n, (name, slope, n)


def test_no_rows():
    """Parameter gradients are zero, nothing else is touched."""
    for gate_rows in (1, 4):
        d = cb.NormDesc.make(0, 64, gate="sigmoid", gate_rows=gate_rows)
        e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
        w = torch.ones(64, device="cuda")
        st = torch.empty((0, 4), device="cuda")
        cb.block_norm_fwd(d, e, e, e, cb.NormParams(w, None, w), e, e, st)
        g = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
        cb.block_norm_bwd(d, e, e, e, cb.NormParams(w, None, w), st, e, e, e, e, e, cb.NormParams(g[0], None, g[1]),
                          cb.norm_workspace(d))
        assert (g[0] == 0).all() and (g[1] == 0).all()


def test_other_stream_and_graph():
    """On a stream of its own, and captured: every replay gives what an eager
    call gives on the inputs of the time."""
    t, p = _draw(900, 264, "rms", "rms", "sigmoid", 300, "bf16", "bf16", False, True, True, 9)
    d = cb.NormDesc.make(900, 264, gate="sigmoid", gate_rows=300, eps=EPS)
    P = {k: None if a is None else a.cuda() for k, a in p.items()}
    params = cb.NormParams(*(P[k] for k in PARAMS))
    x, u, g, dy, dh = (t[k].cuda() for k in ("x", "u", "gate", "dy", "dh"))
    new = lambda: dict(y=torch.zeros_like(x), h=torch.zeros_like(u), st=torch.zeros((900, 4), device="cuda"),  # noqa: E731
                       dx=torch.zeros_like(x), du=torch.zeros_like(u), dg=torch.zeros_like(g),
                       w=torch.zeros(264, device="cuda"), s=torch.zeros(264, device="cuda"), ws=cb.norm_workspace(d))
    a, b = new(), new()
    torch.cuda.synchronize()

    def step(o, stream=None):
        cb.block_norm_fwd(d, x, u, g, params, o["y"], o["h"], o["st"], stream=stream)
        cb.block_norm_bwd(d, o["y"], u, g, params, o["st"], dy, dh, o["dx"], o["du"], o["dg"],
                          cb.NormParams(o["w"], None, None, None, o["s"]), o["ws"], stream=stream)

    s = torch.cuda.Stream()
    step(a, s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(a, torch.cuda.current_stream())
    for k in range(4):
        u.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        step(b)
        torch.cuda.synchronize()
        for n in a:
            if n != "ws":
                assert torch.equal(a[n], b[n]), (k, n)


def test_binding_refuses():
    d = cb.NormDesc.make(4, 64, gate="sigmoid")
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    st = torch.zeros((4, 4), device="cuda")
    ok = dict(x=x, u=x.clone(), gate=x.clone(), y=x.clone(), h=x.clone())
    for bad in (dict(x=x.float()), dict(u=x[:3]), dict(gate=x[:, :32]), dict(h=x.t().contiguous().t())):
        a = {**ok, **bad}
        with pytest.raises(ValueError):
            cb.block_norm_fwd(d, a["x"], a["u"], a["gate"], None, a["y"], a["h"], st)
    with pytest.raises(ValueError):
        cb.NormParams(x)
    with pytest.raises(ValueError):
        cb.block_norm_fwd(d, x, x, x, cb.NormParams(torch.ones(32, device="cuda")), x, x, st)
    for bad in (dict(y=None), dict(h=None), dict(gate=None), dict(u=None)):
        a = {**ok, **bad}
        with pytest.raises(cb.CbwError):
            cb.block_norm_fwd(d, a["x"], a["u"], a["gate"], None, a["y"], a["h"], st)


@pytest.mark.parametrize("rows,C", [(9, 64), (3, 4104), (2, 16384)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_far_out(rows, C, dtype):
    """The sigmoid and its derivative keep their own relative accuracy however
    far out the gate is.  With neither norm nor scale y - x = a u, dgate = dy u
    a', du = dy a.  float32: an exponential (1 ulp), an addition, a division
    and up to five products: 32 * 2^-24.  bf16: its own rounding, and 2^-14 for
    a faster exponential, whose argument is rounded (at most 88 * 1.5 * 2^-24).
    Past 87 the derivative leaves float32's normal range."""
    g = torch.Generator().manual_seed(23)
    gate = torch.cat([torch.linspace(-100, 100, rows * C // 2), 12 * torch.randn(rows * C // 2, generator=g)])
    gate = gate[torch.randperm(rows * C, generator=g)].view(rows, C).to(DT[dtype])
    u, dy = (torch.randn((rows, C), generator=g).to(DT[dtype]) for _ in range(2))
    d = cb.NormDesc.make(rows, C, "none", "none", "sigmoid", 1, dtype, "f32", EPS)
    G, U, DY, x = gate.cuda(), u.cuda(), dy.float().cuda(), torch.zeros((rows, C), device="cuda")
    y, dx, du, dg = torch.empty_like(x), torch.empty_like(x), torch.empty_like(U), torch.empty_like(G)
    st = torch.empty((rows, 4), device="cuda")
    cb.block_norm_fwd(d, x, U, G, None, y, None, st)
    cb.block_norm_bwd(d, y, U, G, None, st, DY, None, dx, du, dg, None, cb.norm_workspace(d))
    near = 32 * ref.U32 if dtype == "f32" else 2.0 ** -14
    a = torch.sigmoid(gate.double())
    da = a * torch.sigmoid(-gate.double())
    for name, got, want in (("y", y, a * u.double()), ("dgate", dg, dy.double() * u.double() * da), ("du", du, dy.double() * a)):
        ref.check(got, want, near * want.abs(), name)


def test_gate_row_for_more_rows_than_there_can_be():
    """gate_rows at the end of its type: one gate row serves all rows, as with gate_rows = rows."""
    rows, C = 300, 72
    t, p = _draw(rows, C, "rms", "rms", "sigmoid", rows, "bf16", "bf16", False, False, True, 24)
    params = cb.NormParams(*(None if p[k] is None else p[k].cuda() for k in PARAMS))
    x, u, g, dy, dh = (t[k].cuda() for k in ("x", "u", "gate", "dy", "dh"))
    outs = []
    for gate_rows in (rows, (1 << 63) - 1):
        d = cb.NormDesc.make(rows, C, gate="sigmoid", gate_rows=gate_rows, eps=EPS)
        y, h, st = torch.empty_like(x), torch.empty_like(u), torch.empty((rows, 4), device="cuda")
        cb.block_norm_fwd(d, x, u, g, params, y, h, st)
        dx, du, dg = torch.empty_like(x), torch.empty_like(u), torch.empty_like(g)
        cb.block_norm_bwd(d, y, u, g, params, st, dy, dh, dx, du, dg, None, cb.norm_workspace(d))
        outs.append((y, h, st, dx, du, dg))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def _statistics_bound(v, err, kind, r):
    """Bounds of what the kernel's mean and r of the rows v (64 bits, each
    value known to within err) may be off by: the mean's from its terms; r's
    relative one is half the mean square's, which changes by at most twice the
    product of the deviations' and the errors' root mean squares."""
    err = err + ref.ROW * v.abs().mean(1, keepdim=True)
    mean = err.mean(1) if kind == "layer" else torch.zeros(v.shape[0], dtype=torch.float64)
    return mean, r * (2 * r * err.square().mean(1).sqrt() + ref.ROW)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")], ids="-".join)
@pytest.mark.parametrize("kinds", [("rms", "rms"), ("layer", "layer"), ("layer", "none"), ("none", "layer"), ("rms", "layer")],
                         ids="-".join)
def test_statistics(size, types, kinds):
    """All four columns: mean and r of y and of u, zeros where there is no norm."""
    rows, C = size
    pre, post = kinds
    print("[case]", rows, C, *kinds, *types, flush=True)
    t, p = _draw(rows, C, pre, post, "linear", 1, *types, True, True, True, 21, 0.5)
    d = cb.NormDesc.make(rows, C, pre, post, "linear", 1, *types, EPS)
    params = cb.NormParams(*(None if p[k] is None else p[k].cuda() for k in PARAMS))
    x, u, g = (t[k].cuda() for k in ("x", "u", "gate"))
    h = None if pre == "none" else torch.empty_like(u)
    st = torch.full((rows, 4), float("nan"), device="cuda")
    cb.block_norm_fwd(d, x, u, g, params, torch.empty_like(x), h, st)
    got = st.cpu().double()
    want = ref.norm_fwd(t["x"], t["u"], t["gate"], p, pre, post, "linear", 1, EPS)
    y, y_err = want["y"]
    for at, v, err, kind, mu, r in ((0, y, y_err, pre, want.get("mu"), want.get("r")),
                                    (2, t["u"].double(), 0 * y, post, want["mu_u"], want["r_u"])):
        if kind == "none":
            assert (got[:, at:at + 2] == 0).all()
            continue
        mean_off, r_off = _statistics_bound(v, err, kind, r[:, 0])
        assert ((got[:, at] - mu[:, 0]).abs() <= mean_off).all(), "mean"
        assert ((got[:, at + 1] - r[:, 0]).abs() <= r_off).all(), "r"


@pytest.mark.parametrize("C", [136, 520, 2056, 8200, 16384])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pre,post", [("rms", "rms"), ("layer", "layer"), ("rms", "layer")])
def test_backward_from_the_forward_statistics(C, dtype, pre, post):
    """A step as a program makes it: the backward pass reads the statistics
    that the forward pass wrote.  The stream is float32, so that y is stored to
    within the bounds' own size."""
    rows = 5
    t, p = _draw(rows, C, pre, post, "sigmoid", 1, dtype, "f32", True, True, True, 22, 0.25)
    d = cb.NormDesc.make(rows, C, pre, post, "sigmoid", 1, dtype, "f32", EPS)
    P = {k: v.cuda() for k, v in p.items()}
    params = cb.NormParams(*(P[k] for k in PARAMS))
    x, u, g, dy, dh = (t[k].cuda() for k in ("x", "u", "gate", "dy", "dh"))
    y, h, st = torch.empty_like(x), torch.empty_like(u), torch.full((rows, 4), float("nan"), device="cuda")
    cb.block_norm_fwd(d, x, u, g, params, y, h, st)
    grads = {k: torch.full_like(v, float("nan")) for k, v in P.items()}
    dx, du, dg = torch.empty_like(x), torch.empty_like(u), torch.empty_like(g)
    cb.block_norm_bwd(d, y, u, g, params, st, dy, dh, dx, du, dg, cb.NormParams(*(grads[k] for k in PARAMS)),
                      cb.norm_workspace(d))
    want = ref.norm_bwd(y, t["u"], t["gate"], p, t["dy"], t["dh"], pre, post, "sigmoid", 1, EPS)
    for name, got in (("dx", dx), ("du", du), ("dgate", dg), *grads.items()):
        ref.check(got, *want[name], name)
