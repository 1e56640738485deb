"""The gated layer's products and their gradients against 64 bits: every kind of
group lengths, widths that fill no tile, strides, both types, all activations."""
import pytest
import torch

import block_ref as ref
import gated_ref as gref
import paper_2109_07710_amd as cb
from test_gpu_experts import CASES, _lengths, _outside, _rows

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _draw(off, rows, C, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    E = len(off) - 1
    x = torch.randn((rows, C), generator=g).to(DT[dtype])
    w = (torch.randn((E, 2, K, C), generator=g) * (2.0 / C) ** 0.5).to(DT[dtype])
    dy = torch.randn((rows, C), generator=g).to(DT[dtype])
    w2 = (torch.randn((E, C, K), generator=g) / K ** 0.5).to(DT[dtype])
    gu = (1.5 * torch.randn((rows, 2 * K), generator=g)).to(DT[dtype])
    return x, w, dy, w2, gu


def _off(off):
    return torch.tensor(off, dtype=torch.int32, device="cuda")


def _nan(rows, n, dtype, stride=None):
    return _rows(torch.full((rows, n), float("nan"), dtype=DT[dtype]), n if stride is None else stride)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", range(len(CASES)), ids=lambda i: "E%d_r%d_C%d_K%d" % (len(CASES[i][0]) - 1, *CASES[i][1:]))
def test_products(at, dtype):
    off, rows, C, K = CASES[at]
    print("[case]", dtype, rows, C, K, flush=True)
    x, w, dy, w2, gu = _draw(off, rows, C, K, dtype, at)
    xs, hs, gs = C + 16, K + 24, 2 * K + 8
    o, inside = _off(off), slice(off[0], off[-1])
    # the rows of no expert hold NaN: they must not reach any result
    own = torch.zeros(rows, 1, dtype=torch.bool)
    own[inside] = True
    X, dY, G = (_rows(torch.where(own, t, float("nan")), s) for t, s in ((x, xs), (dy, xs), (gu, gs)))
    W, W2 = w.cuda(), w2.cuda()
    for act in gref.ACTS:
        d = cb.GatedDesc.make(len(off) - 1, rows, C, K, act, dtype, xs, hs, gs)
        H, GU = _nan(rows, K, dtype, hs), _nan(rows, 2 * K, dtype, gs)
        cb.expert_gated_fwd(d, X, W, o, H, GU)
        want = gref.forward(x, w, off, act)
        for name, got in (("h", H), ("gu", GU)):
            ref.check(got[inside], want[name][0][inside], want[name][1][inside], act + " " + name)
            _outside(got, off, name)
        alone = _nan(rows, K, dtype, hs)
        cb.expert_gated_fwd(d, X, W, o, alone)
        assert torch.equal(alone[inside], H[inside]), "H beside GU and without"
        dGU, again = _nan(rows, 2 * K, dtype, gs), _nan(rows, K, dtype, hs)
        cb.expert_gated_bwd(d, dY, W2, o, G, dGU, again)
        want = gref.backward(dy, w2, gu, off, act)
        for name, got in (("dgu", dGU), ("h", again)):
            ref.check(got[inside], want[name][0][inside], want[name][1][inside], act + " " + name)
            _outside(got, off, name)
        place = _rows(torch.where(own, gu, float("nan")), gs)
        cb.expert_gated_bwd(d, dY, W2, o, place, place)
        assert torch.equal(place[inside], dGU[inside]), "in place, without H"
        _outside(place, off, "in place")


# (experts, rows, C, K, type): sizes at which the large tiles run, several of
# them to a workgroup, with one, two and more steps and a last one that is short
LARGE = [
    (4, 9000, 64, 2064, "bf16"),
    (4, 9000, 72, 4104, "bf16"),
    (5, 8000, 264, 2128, "bf16"),
    (2, 4000, 72, 4104, "bf16"),       # tiles of 192 rows
    (3, 4100, 136, 4104, "bf16"),
    (20, 2000, 200, 2056, "bf16"),     # tiles of 128 rows
    (20, 2000, 136, 4104, "bf16"),
    (3, 2000, 1032, 264, "bf16"),      # few tiles: rows by 64
    (6, 5001, 72, 1032, "f32"),        # float32 tiles
    (100, 3000, 264, 264, "bf16"),     # more experts than lanes
    (100, 3000, 132, 264, "f32"),
    (80, 4000, 132, 264, "f32"),
]


@pytest.mark.parametrize("at", range(len(LARGE)), ids=lambda i: "E%d_r%d_C%d_K%d_%s" % LARGE[i])
def test_large_tiles(at):
    E, rows, C, K, dtype = LARGE[at]
    act = gref.ACTS[1 + at % 3]
    print("[case]", E, rows, C, K, dtype, act, flush=True)
    off = _lengths(E, rows, 3)
    x, w, dy, w2, gu = _draw(off, rows, C, K, dtype, 7)
    d = cb.GatedDesc.make(E, rows, C, K, act, dtype)
    H, GU, dGU, again = (_nan(rows, n * K, dtype) for n in (1, 2, 2, 1))
    cb.expert_gated_fwd(d, x.cuda(), w.cuda(), _off(off), H, GU)
    cb.expert_gated_bwd(d, dy.cuda(), w2.cuda(), _off(off), gu.cuda(), dGU, again)
    want = gref.forward(x, w, off, act)
    ref.check(H, *want["h"], "h")
    ref.check(GU, *want["gu"], "gu")
    want = gref.backward(dy, w2, gu, off, act)
    ref.check(dGU, *want["dgu"], "dgu")
    ref.check(again, *want["h"], "h again")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", gref.ACTS)
def test_far_values(act, dtype):
    """Pre-activations of every size: the derivatives stay what they tend to, and the sigmoid keeps its accuracy far out."""
    edge = [0.0, -0.0, 1e-30, -1e-30, 1e-3, -1.25, 9.0, -9.0, 20.0, -20.0, 80.0, -80.0, 109.0, -109.0, 111.0, -111.0, 300.0, -300.0,
            1e4, -1e4, 1e13, -1e13, 1e20, -1e20, 1e30, -1e30]
    g = torch.tensor(edge + [0.5] * (-len(edge) % 8)).to(DT[dtype])
    K = g.numel()
    u = torch.linspace(-2, 2, K).to(DT[dtype])
    gu = torch.cat((g, u))[None]
    dy, w2 = torch.ones((1, 8)).to(DT[dtype]), torch.full((1, 8, K), 0.125).to(DT[dtype])   # dH = 1
    d = cb.GatedDesc.make(1, 1, 8, K, act, dtype)
    dGU, H = _nan(1, 2 * K, dtype), _nan(1, K, dtype)
    cb.expert_gated_bwd(d, dy.cuda(), w2.cuda(), _off([0, 1]), gu.cuda(), dGU, H)
    # past 300 the 64-bit form would overflow itself (0 * inf): it stands still there too
    near = gu.double().clamp(-300, 300)
    near[:, K:] = gu[:, K:].double()
    want = gref.backward(dy, w2, near, [0, 1], act)
    big = gu[:, :K].double().clamp(min=300.0) if act in ("relu", "silu", "gelu") else None
    value, bound = (t.clone() for t in want["dgu"])
    h, mh = (t.clone() for t in want["h"])
    if big is not None:
        far = gu[:, :K].double() > 300
        value[:, K:][far] = big[far]
        h[far] = (big * u.double())[far]
        bound[:, K:][far], mh[far] = 4 * gref.U32 * big[far], 4 * gref.U32 * (big * u.double()).abs()[far]
    ref.check(dGU, value, bound, "dgu")
    ref.check(H, h, mh, "h")


def test_infinities_and_nan_stay_in_their_row_and_feature():
    """act(inf) = inf or 1, act(-inf) = 0 and their slopes 1 and 0; a NaN reaches its own values alone (relu: none)."""
    K = 16
    for act in gref.ACTS:
        d = cb.GatedDesc.make(1, 3, 8, K, act, "f32")
        gu = torch.ones((3, 2 * K), device="cuda")
        gu[1, 2], gu[1, 5], gu[1, 9] = float("inf"), float("-inf"), float("nan")
        dy, w2 = torch.ones((3, 8), device="cuda"), torch.full((1, 8, K), 0.125, device="cuda")
        dGU = torch.full((3, 2 * K), 7.0, device="cuda")
        cb.expert_gated_bwd(d, dy, w2, _off([0, 3]), gu, dGU)
        r = dGU.cpu()
        assert r[1, 2] == (0.0 if act == "sigmoid" else 1.0) and r[1, K + 2] == (1.0 if act == "sigmoid" else float("inf")), act
        assert r[1, 5] == 0.0 and r[1, K + 5] == 0.0, act
        assert (r[1, 9] == 0.0 if act == "relu" else torch.isnan(r[1, 9])), act
        r[1, [2, 5, 9, K + 2, K + 5, K + 9]] = r[0, 0]
        same = torch.ones(3, 2 * K, dtype=torch.bool)
        same[1, [2, 5, 9, K + 2, K + 5, K + 9]] = False
        assert torch.equal(r[same], r[0].expand(3, -1)[same]), act


@pytest.mark.parametrize("act", gref.ACTS)
def test_gradient_against_differences(act):
    """dg and du against central differences of sum(dH * H) in 64 bits: third derivatives are below 4 here, so that a step of
    2^-10 leaves 4 / 6 2^-20 |dH u|; and the kernel's own bound.  (relu: values away from the bend.)"""
    g = torch.Generator().manual_seed(2)
    rows, C, K = 9, 16, 24
    off = [0, 4, 9]
    _, _, dy, w2, gu = _draw(off, rows, C, K, "f32", 3)
    if act == "relu":
        gu[:, :K] += 0.01 * torch.sign(gu[:, :K])
    d = cb.GatedDesc.make(2, rows, C, K, act, "f32")
    dGU = _nan(rows, 2 * K, "f32")
    cb.expert_gated_bwd(d, dy.cuda(), w2.cuda(), _off(off), gu.cuda(), dGU)
    dh = torch.cat([dy[a:b].double() @ w2[e].double() for e, (a, b) in enumerate(zip(off, off[1:]))])
    step, G = 2.0 ** -10, gu.double()
    loss = lambda v: dh * gref.act(act, v[:, :K])[0] * v[:, K:]  # noqa: E731
    parts = []
    for half in (0, 1):
        e = torch.zeros_like(G)
        e[:, half * K:(half + 1) * K] = step
        parts.append((loss(G + e) - loss(G - e)) / (2 * step))
    bound = gref.backward(dy, w2, gu, off, act)["dgu"][1] + torch.cat((dh * G[:, K:], 0 * dh), 1).abs() * 2.0 ** -20 + 2.0 ** -40
    ref.check(dGU, torch.cat(parts, 1), bound, "differences")


@pytest.mark.parametrize("dtype,rows", [("bf16", 5), ("bf16", 3000), ("f32", 700)])
def test_captured_and_on_another_stream(dtype, rows):
    """Both calls in a graph, replayed with other inputs and other lengths between eager calls; bit for bit the eager results."""
    E, C, K = 3, 136, 1032
    d = cb.GatedDesc.make(E, rows, C, K, "silu", dtype)
    sets = [_draw([0] * (E + 1), rows, C, K, dtype, s) for s in range(3)]
    offs = [[0, rows // 3, rows // 2, rows], [0, 0, rows, rows], [0, rows, rows, rows]]
    x, w, dy, w2, _ = (t.cuda() for t in sets[0])
    o = _off(offs[0])
    H, GU, dGU = (_nan(rows, n * K, dtype) for n in (1, 2, 2))

    def step(h, gu, dgu):
        cb.expert_gated_fwd(d, x, w, o, h, gu)
        cb.expert_gated_bwd(d, dy, w2, o, gu, dgu)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(H, GU, dGU)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(H, GU, dGU)
    for k in (1, 2, 0, 1):
        for dst, src in zip((x, w, dy, w2), sets[k]):
            dst.copy_(src)
        o.copy_(_off(offs[k]))
        H.fill_(7.0), GU.fill_(7.0), dGU.fill_(7.0)
        graph.replay()
        eager = [torch.full_like(t, 7.0) for t in (H, GU, dGU)]
        step(*eager)
        torch.cuda.synchronize()
        for got, want in zip((H, GU, dGU), eager):
            assert torch.equal(got, want)


@pytest.mark.parametrize("E,K", [(1, 2064), (64, 72)])
def test_rows_past_32_bits(E, K):
    """Rows so far apart that their addresses pass 2^32 elements: bit for bit what adjacent ones give, large tiles and streaming."""
    rows, C, far = 4400, 64, (1 << 20) - 8
    off = _lengths(E, rows, 4) if E > 1 else [0, rows]
    x, w, dy, w2, _ = (t.cuda() for t in _draw(off, rows, C, K, "bf16", 8))
    o = _off(off)
    near = cb.GatedDesc.make(E, rows, C, K)
    H, GU, dGU = (_nan(rows, n * K, "bf16") for n in (1, 2, 2))
    cb.expert_gated_fwd(near, x, w, o, H, GU)
    cb.expert_gated_bwd(near, dy, w2, o, GU, dGU)
    d = cb.GatedDesc.make(E, rows, C, K, x_stride=far, h_stride=far, gu_stride=far)
    space = [torch.empty(rows * far, dtype=torch.bfloat16, device="cuda").view(rows, far) for _ in range(3)]
    X, h, gu = space[0][:, :C], space[1][:, :K], space[2][:, :2 * K]
    X.copy_(x)
    cb.expert_gated_fwd(d, X, w, o, h, gu)
    assert torch.equal(h, H) and torch.equal(gu, GU)
    X.copy_(dy)
    cb.expert_gated_bwd(d, X, w2, o, gu, gu)
    assert torch.equal(gu, dGU)


def test_offsets_without_sense_stay_inside():
    """Decreasing and out-of-range offsets: nothing outside the rows is written, and the call ends."""
    rows, C, K = 300, 64, 128
    d = cb.GatedDesc.make(4, rows, C, K, "silu", "bf16")
    x, w, dy, w2, gu = (t.cuda() for t in _draw([0] * 5, rows, C, K, "bf16", 1))
    for off in ([0, 200, 100, 250, 300], [-50, 20, 100, 900, 2000], [300, 0, 300, 0, 300], [2 ** 31 - 1, -2 ** 31, 5, 5, 9]):
        guard = [torch.full((rows + 64, n), 7.0, dtype=torch.bfloat16, device="cuda") for n in (K, 2 * K, 2 * K)]
        h, g2, dg = (t[32:32 + rows] for t in guard)
        cb.expert_gated_fwd(d, x, w, _off(off), h, g2)
        cb.expert_gated_bwd(d, dy, w2, _off(off), gu, dg)
        torch.cuda.synchronize()
        for t in guard:
            assert bool((t[:32] == 7).all()) and bool((t[32 + rows:] == 7).all()), off


def test_whole_layer_with_the_other_calls():
    """Forward, the next filter, and every gradient with the calls that stand beside these, against autograd in 64 bits.
    float32: each of the five products and the activations leaves some 2^-20 of a result's size; 2^-14 in the 2-norm."""
    off, rows, C, K = [0, 5, 5, 140, 201], 201, 72, 104
    E = len(off) - 1
    x, w, dy, w2, _ = _draw(off, rows, C, K, "f32", 5)
    X, W, dY, W2, o = x.cuda(), w.cuda(), dy.cuda(), w2.cuda(), _off(off)
    d = cb.GatedDesc.make(E, rows, C, K, "silu", "f32")
    first, second = cb.ExpertDesc.make(E, rows, C, 2 * K, "f32"), cb.ExpertDesc.make(E, rows, K, C, "f32")
    ws = torch.empty(max(cb.cbw_expert_workspace_size(first), cb.cbw_expert_workspace_size(second), 1), dtype=torch.uint8, device="cuda")
    new = lambda *n: torch.full(n, float("nan"), device="cuda")  # noqa: E731
    H, GU, Y, dX, dW, dW2 = new(rows, K), new(rows, 2 * K), new(rows, C), new(rows, C), new(E, 2 * K, C), new(E, C, K)
    cb.expert_gated_fwd(d, X, W, o, H, GU)
    cb.expert_fwd(second, H, W2, o, Y, None, ws)
    H.fill_(float("nan"))
    cb.expert_gated_bwd(d, dY, W2, o, GU, GU, H)                 # in place, H once more
    cb.expert_bwd_weight(second, H, dY, o, dW2, ws)
    cb.expert_bwd_weight(first, X, GU, o, dW, ws)
    cb.expert_bwd_data(first, GU, W.view(E, 2 * K, C), o, None, dX, ws)
    x64, w64, v64 = (t.double().requires_grad_() for t in (x, w, w2))
    y64 = torch.cat([(torch.nn.functional.silu(x64[a:b] @ w64[e, 0].t()) * (x64[a:b] @ w64[e, 1].t())) @ v64[e].t()
                     for e, (a, b) in enumerate(zip(off, off[1:]))])
    (y64 * dy.double()).sum().backward()
    for name, got, want in (("Y", Y, y64.detach()), ("dX", dX, x64.grad), ("dW", dW.view_as(w), w64.grad), ("dW2", dW2, v64.grad)):
        err = float((got.cpu().double() - want).norm() / want.norm())
        assert err <= 2.0 ** -14, (name, err)
