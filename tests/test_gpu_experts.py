"""Products grouped by expert against 64 bits: every kind of group lengths,
widths that fill no tile, strides, footprints, both types."""
import numpy as np
import pytest
import torch

import block_ref as ref
import paper_2109_07710_amd as cb

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _rows(t, stride, fill=float("nan")):
    """The rows on the device, `stride` elements apart in a larger buffer."""
    buf = torch.full((t.shape[0], stride), fill, dtype=t.dtype, device="cuda")
    v = buf[:, :t.shape[1]]
    v.copy_(t)
    return v


def _draw(off, rows, C, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    E = len(off) - 1
    x = torch.randn((rows, C), generator=g).to(DT[dtype])
    w = (torch.randn((E, K, C), generator=g) / C ** 0.5).to(DT[dtype])
    dy = torch.randn((rows, K), generator=g).to(DT[dtype])
    live = torch.rand((rows, C), generator=g) < 0.4
    return x, w, dy, live


def _outside(got, off, what):
    """Rows of no expert keep what they held."""
    r = torch.ones(got.shape[0], dtype=torch.bool)
    r[off[0]:off[-1]] = False
    assert torch.isnan(got.float().cpu()[r]).all(), what + ": rows of no expert were written"


# (offsets, rows, C, K)
CASES = [
    ([0, 1], 1, 8, 8),
    ([0, 1], 1, 64, 256),
    ([0, 0, 3, 3, 5], 5, 72, 104),
    ([0, 300], 300, 200, 136),
    ([0, 17, 17, 300, 301, 556, 557], 557, 264, 520),
    ([3, 40, 90], 100, 96, 64),                 # rows before and after the experts' own
    ([0, 0, 0], 4, 64, 64),                     # nobody has a row
    ([0, 64, 128, 256, 512], 512, 128, 256),    # whole tiles
    ([0, 5, 1300], 1300, 40, 72),
    (list(range(0, 71)), 70, 64, 32),           # more experts than lanes, a row each
    ([0] * 100 + [33] * 31, 33, 32, 96),        # empty experts before and behind
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "E%d_r%d_C%d_K%d" % (len(c[0]) - 1, c[1], c[2], c[3]))
def test_products(case, dtype):
    off, rows, C, K = case
    print("[case]", dtype, rows, C, K, flush=True)
    x, w, dy, live = _draw(off, rows, C, K, dtype, 1)
    xs, ys = C + 16, K + 24
    d = cb.ExpertDesc.make(len(off) - 1, rows, C, K, dtype, xs, ys)
    ws = cb.expert_workspace(d)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    # the rows of no expert hold NaN: they must not reach any result
    own = torch.zeros(rows, 1, dtype=torch.bool)
    own[off[0]:off[-1]] = True
    X = _rows(torch.where(own, x, float("nan")), xs)
    dY = _rows(torch.where(own, dy, float("nan")), ys)
    W = w.cuda()
    nan = lambda n, m, s: _rows(torch.full((n, m), float("nan"), dtype=DT[dtype]), s)  # noqa: E731
    inside = slice(off[0], off[-1])
    for relu in (False, True):
        Y = nan(rows, K, ys)
        mask = torch.zeros((rows * K + 31) // 32, dtype=torch.int32, device="cuda") if relu and K % 32 == 0 else None
        cb.expert_fwd(d, X, W, o, Y, mask, ws, cb.CBW_FLAG_RELU if relu else 0)
        y, m = ref.expert_fwd(x, w, off, relu)
        ref.check(Y[inside], y[inside], m[inside], "Y")
        _outside(Y, off, "Y")
        if mask is not None:
            want = torch.zeros((rows, K), dtype=torch.bool)
            want[inside] = Y.cpu()[inside] > 0
            assert torch.equal(mask.cpu(), ref.bits(want)), "footprint"
    for lv in (None, live):
        dX = nan(rows, C, xs)
        cb.expert_bwd_data(d, dY, W, o, None if lv is None else ref.bits(lv).cuda(), dX, ws)
        dx, m = ref.expert_bwd_data(dy, w, off, lv)
        ref.check(dX[inside], dx[inside], m[inside], "dX")
        _outside(dX, off, "dX")
        if lv is not None:
            dead = dX.cpu()[inside][~lv[inside]]
            assert (dead.view(torch.int16 if dtype == "bf16" else torch.int32) == 0).all(), "dead values are +0.0"
    dW = torch.full((len(off) - 1, K, C), float("nan"), device="cuda")
    cb.expert_bwd_weight(d, X, dY, o, dW, ws)
    dw, m = ref.expert_bwd_weight(x, dy, off)
    ref.check(dW, dw, m, "dW")


def _lengths(E, rows, seed):
    """Uneven group lengths that add up to `rows`, the second group empty."""
    g = torch.Generator().manual_seed(seed)
    p = torch.exp(torch.randn(E, generator=g))
    p[1] = 0.0
    n = torch.floor(p / p.sum() * rows).long()
    n[0] += rows - n.sum()
    return [0] + n.cumsum(0).tolist()


# (experts, rows, the output's features, the reduction's, type): sizes at
# which the large tiles run, several of them to a workgroup, with one, two and
# more reduction steps and a last one that is short
LARGE = [
    (4, 9000, 4128, 64, "bf16"),       # 256 x 256 tiles, one step
    (4, 9000, 4104, 72, "bf16"),       # two
    (5, 8000, 4128, 264, "bf16"),      # five
    (20, 2000, 4104, 200, "bf16"),     # 128 x 128 tiles
    (3, 2000, 264, 1032, "bf16"),      # few tiles: rows by 64
    (6, 5001, 1032, 72, "f32"),        # 64 x 64 tiles
    (100, 3000, 264, 264, "bf16"),     # more experts than lanes
    (100, 3000, 264, 132, "f32"),
]


@pytest.mark.parametrize("E,rows,P,R,dtype", LARGE)
def test_large_tiles(E, rows, P, R, dtype):
    print("[case]", E, rows, P, R, dtype, flush=True)
    off = _lengths(E, rows, 3)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    x, w, _, _ = _draw(off, rows, R, P, dtype, 7)
    d = cb.ExpertDesc.make(E, rows, R, P, dtype)
    Y = torch.full((rows, P), float("nan"), dtype=DT[dtype], device="cuda")
    mask = torch.zeros((rows * P + 31) // 32, dtype=torch.int32, device="cuda") if P % 32 == 0 else None
    cb.expert_fwd(d, x.cuda(), w.cuda(), o, Y, mask, cb.expert_workspace(d), cb.CBW_FLAG_RELU)
    ref.check(Y, *ref.expert_fwd(x, w, off, True), "Y")
    if mask is not None:
        assert torch.equal(mask.cpu(), ref.bits(Y.cpu() > 0)), "footprint"
    # the data gradient with as many features to write and as many to reduce
    _, w, dy, live = _draw(off, rows, P, R, dtype, 8)
    d = cb.ExpertDesc.make(E, rows, P, R, dtype)
    for lv in (None, live):
        dX = torch.full((rows, P), float("nan"), dtype=DT[dtype], device="cuda")
        cb.expert_bwd_data(d, dy.cuda(), w.cuda(), o, None if lv is None else ref.bits(lv).cuda(), dX, cb.expert_workspace(d))
        ref.check(dX, *ref.expert_bwd_data(dy, w, off, lv), "dX")


@pytest.mark.parametrize("E,rows,C,K,dtype", [(5, 2501, 2056, 2056, "bf16"), (3, 9000, 520, 264, "bf16"), (70, 1500, 264, 520, "bf16"),
                                              (5, 3001, 264, 520, "f32"), (64, 4000, 520, 136, "bf16")])
def test_large_weight_gradients(E, rows, C, K, dtype):
    """Several tiles to a workgroup, experts in order of their lengths, split and whole ones side by side."""
    print("[case]", E, rows, C, K, dtype, flush=True)
    off = _lengths(E, rows, 4)
    x, _, dy, _ = _draw(off, rows, C, K, dtype, 9)
    d = cb.ExpertDesc.make(E, rows, C, K, dtype)
    ws = cb.expert_workspace(d)
    ws.fill_(255)
    dW = torch.full((E, K, C), float("nan"), device="cuda")
    cb.expert_bwd_weight(d, x.cuda(), dy.cuda(), torch.tensor(off, dtype=torch.int32, device="cuda"), dW, ws)
    ref.check(dW, *ref.expert_bwd_weight(x, dy, off), "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_split_experts(dtype):
    """Experts whose rows are taken in several parts, between ones that are
    not, twice over a workspace that held other sums: the same bits."""
    off = [0, 2100, 2100, 2101, 5400, 6000]
    x, w, dy, _ = _draw(off, 6000, 72, 40, dtype, 2)
    d = cb.ExpertDesc.make(5, 6000, 72, 40, dtype)
    n = cb.cbw_expert_workspace_size(d)
    assert n > 0
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    got = []
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        dW = torch.full((5, 40, 72), float("nan"), device="cuda")
        cb.expert_bwd_weight(d, x.cuda(), dy.cuda(), o, dW, ws)
        got.append(dW)
    assert torch.equal(*got)
    ref.check(got[0], *ref.expert_bwd_weight(x, dy, off), "dW")


def test_gradients_are_differences():
    """The products are bilinear: L = sum(Y G) changes by exactly <dX, v> and
    <dW, v> along any v.  float32: the difference's rounding is what remains."""
    off = [0, 9, 9, 50]
    x, w, g, _ = _draw(off, 50, 40, 24, "f32", 3)
    d = cb.ExpertDesc.make(3, 50, 40, 24, "f32")
    ws, o = cb.expert_workspace(d), torch.tensor(off, dtype=torch.int32, device="cuda")
    X, W, G = x.cuda(), w.cuda(), g.cuda()

    def loss(X, W):
        Y = torch.empty_like(G)
        cb.expert_fwd(d, X, W, o, Y, None, ws)
        return float((Y.double() * G.double()).sum())

    dX, dW = torch.empty_like(X), torch.empty_like(W)
    cb.expert_bwd_data(d, G, W, o, None, dX, ws)
    cb.expert_bwd_weight(d, X, G, o, dW, ws)
    for grad, at in ((dX, 0), (dW, 1)):
        v = grad / grad.norm()
        plus = loss(X + v, W) if at == 0 else loss(X, W + v)
        minus = loss(X - v, W) if at == 0 else loss(X, W - v)
        want = float((grad.double() * v.double()).sum())
        assert abs((plus - minus) / 2 - want) <= 1e-4 * want


def test_nonfinite_rows_stay_in_their_row():
    """An infinity in one row of X reaches that row of Y alone, and the other
    experts' dW not at all."""
    off = [0, 20, 33, 60]
    x, w, dy, _ = _draw(off, 60, 64, 64, "bf16", 4)
    x[21, 5] = float("inf")
    d = cb.ExpertDesc.make(3, 60, 64, 64)
    ws, o = cb.expert_workspace(d), torch.tensor(off, dtype=torch.int32, device="cuda")
    Y = torch.empty((60, 64), dtype=torch.bfloat16, device="cuda")
    cb.expert_fwd(d, x.cuda(), w.cuda(), o, Y, None, ws)
    fine = torch.isfinite(Y).all(1).cpu()
    assert not fine[21] and fine.sum() == 59
    dW = torch.empty((3, 64, 64), device="cuda")
    cb.expert_bwd_weight(d, x.cuda(), dy.cuda(), o, dW, ws)
    assert torch.isfinite(dW[0]).all() and torch.isfinite(dW[2]).all() and not torch.isfinite(dW[1]).all()


def test_bad_offsets_stay_in_bounds():
    """Offsets out of range and decreasing: no output row or buffer outside is
    touched (guard rows around the tensors), whatever the values are."""
    rows, C, K = 40, 64, 64
    d = cb.ExpertDesc.make(4, rows, C, K)
    ws = cb.expert_workspace(d)
    for off in ([-5, 10, 1000, 7, 40], [40, 0, 40, 0, 40], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        o = torch.tensor(off, dtype=torch.int64).to(torch.int32).cuda()
        X = torch.randn((rows, C), device="cuda").bfloat16()
        W = torch.randn((4, K, C), device="cuda").bfloat16()
        buf = torch.full((rows + 64, K), 7.0, dtype=torch.bfloat16, device="cuda")
        cb.expert_fwd(d, X, W, o, buf[32:32 + rows], None, ws)
        cb.expert_bwd_data(d, X, W, o, None, buf[32:32 + rows], ws)
        dW = torch.full((6, K, C), 7.0, device="cuda")
        cb.expert_bwd_weight(d, X, X, o, dW[1:5], ws)
        torch.cuda.synchronize()
        assert (buf[:32] == 7).all() and (buf[32 + rows:] == 7).all() and (dW[0] == 7).all() and (dW[5] == 7).all()


def test_no_rows():
    d = cb.ExpertDesc.make(3, 0, 64, 32)
    ws, o = cb.expert_workspace(d), torch.zeros(4, dtype=torch.int32, device="cuda")
    e = lambda m: torch.empty((0, m), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    W = torch.randn((3, 32, 64), device="cuda").bfloat16()
    cb.expert_fwd(d, e(64), W, o, e(32), None, ws)
    cb.expert_bwd_data(d, e(32), W, o, None, e(64), ws)
    dW = torch.full((3, 32, 64), 5.0, device="cuda")
    cb.expert_bwd_weight(d, e(64), e(32), o, dW, ws)
    assert (dW == 0).all()


def test_rows_past_2_31_elements():
    """Row tensors of more than 2^31 elements (a row stride of 2^19): the last
    rows, alone in their expert, are those that are asked for."""
    rows, C, K, stride = 4200, 64, 32, 1 << 19
    x = torch.empty((rows, stride), dtype=torch.bfloat16, device="cuda")[:, :C]
    g = torch.Generator(device="cuda").manual_seed(5)
    x.copy_(torch.randn((rows, C), generator=g, device="cuda"))
    w = (torch.randn((2, K, C), generator=g, device="cuda") / 8).bfloat16()
    dy = torch.randn((rows, K), generator=g, device="cuda").bfloat16()
    off = [0, 4190, 4200]
    d = cb.ExpertDesc.make(2, rows, C, K, "bf16", stride, K)
    ws, o = cb.expert_workspace(d), torch.tensor(off, dtype=torch.int32, device="cuda")
    Y = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda")
    cb.expert_fwd(d, x, w, o, Y, None, ws)
    y, m = ref.expert_fwd(x.cpu(), w.cpu(), off, False)
    ref.check(Y, y, m, "Y")
    dW = torch.empty((2, K, C), device="cuda")
    cb.expert_bwd_weight(d, x, dy, o, dW, ws)
    ref.check(dW, *ref.expert_bwd_weight(x.cpu(), dy.cpu(), off), "dW")
    dX = x
    cb.expert_bwd_data(d, dy, w, o, None, dX, ws)
    dx, m = ref.expert_bwd_data(dy.cpu(), w.cpu(), off, None)
    ref.check(dX, dx, m, "dX")


def test_other_stream_and_graph():
    """On a stream of its own, and captured: the graph's replays follow the
    offsets and rows that its tensors hold at the time."""
    off = [[0, 100, 300], [0, 300, 300], [0, 7, 9]]
    x, w, dy, _ = _draw([0, 100, 300], 300, 128, 64, "bf16", 6)
    d = cb.ExpertDesc.make(2, 300, 128, 64)
    s = torch.cuda.Stream()
    ws = cb.expert_workspace(d)
    X, W, dY, o = x.cuda(), w.cuda(), dy.cuda(), torch.tensor(off[0], dtype=torch.int32, device="cuda")
    Y = torch.zeros((300, 64), dtype=torch.bfloat16, device="cuda")
    dW = torch.zeros((2, 64, 128), device="cuda")
    torch.cuda.synchronize()

    def step(stream):
        cb.expert_fwd(d, X, W, o, Y, None, ws, stream=stream)
        cb.expert_bwd_weight(d, X, dY, o, dW, ws, stream=stream)

    step(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(torch.cuda.current_stream())
    for k, want in enumerate(off + off):
        o.copy_(torch.tensor(want, dtype=torch.int32))
        X.copy_(x * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        xs = (x * (k + 1)).to(torch.bfloat16)
        y, m = ref.expert_fwd(xs, w, want, False)
        n = want[-1]
        ref.check(Y[:n], y[:n], m[:n], "Y")
        ref.check(dW, *ref.expert_bwd_weight(xs, dy, want), "dW")


def test_binding_refuses():
    d = cb.ExpertDesc.make(2, 10, 64, 32)
    ws, o = cb.expert_workspace(d), torch.zeros(3, dtype=torch.int32, device="cuda")
    X = torch.zeros((10, 64), dtype=torch.bfloat16, device="cuda")
    Y = torch.zeros((10, 32), dtype=torch.bfloat16, device="cuda")
    W = torch.zeros((2, 32, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (dict(X=X.float()), dict(X=X[:9]), dict(X=torch.zeros((10, 80), dtype=torch.bfloat16, device="cuda")[:, :64]),
                dict(W=W[:1]), dict(W=W.transpose(1, 2)), dict(o=o.long()), dict(o=o[:2]), dict(Y=Y.cpu())):
        a = dict(X=X, W=W, o=o, Y=Y, **{})
        a.update(bad)
        with pytest.raises(ValueError):
            cb.expert_fwd(d, a["X"], a["W"], a["o"], a["Y"], None, ws)
    with pytest.raises(cb.CbwError):
        cb.expert_fwd(d, X, W, o, Y, torch.zeros(10, dtype=torch.int32, device="cuda"), ws)   # a footprint without ReLU
    with pytest.raises(cb.CbwError):
        cb.expert_fwd(d, X, W, o, Y, None, ws, 1)
    big = cb.ExpertDesc.make(2, 100000, 64, 32)
    t = lambda m: torch.zeros((100000, m), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    with pytest.raises(cb.CbwError) as e:
        cb.expert_bwd_weight(big, t(64), t(32), o, torch.zeros((2, 32, 64), device="cuda"), ws[:0])
    assert e.value.status == cb.CBW_ERR_WORKSPACE


@pytest.mark.parametrize("product", ["forward", "data"])
def test_more_workgroups_than_one_axis_takes(product):
    """A row for each of 1024 experts, by so many features that over 2^24
    workgroups of 256 threads are launched: 2^32 threads, more than a launch
    has along one axis."""
    P, R, E = (1 << 20) - 8, 8, 1024
    o = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(13)
    x = torch.randn((E, R), generator=g, device="cuda").bfloat16()
    fwd = product == "forward"
    w = torch.empty((E, P, R) if fwd else (E, R, P), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = torch.full((E, P), float("nan"), dtype=torch.bfloat16, device="cuda")
    if fwd:
        d = cb.ExpertDesc.make(E, E, R, P)
        cb.expert_fwd(d, x, w, o, out, None, cb.expert_workspace(d))
    else:
        d = cb.ExpertDesc.make(E, E, P, R)
        cb.expert_bwd_data(d, x, w, o, None, out, cb.expert_workspace(d))
    assert not any(bool(v.isnan().any()) for v in out.split(64)), "values were not written"
    for e in (0, 63, 64, 500, 1023):
        we, xe = (w[e].t() if fwd else w[e]).cpu().double(), x[e:e + 1].cpu().double()
        ref.check(out[e:e + 1], xe @ we, (R + 4) * ref.U32 * (xe.abs() @ we.abs()), "expert %d" % e)


def _part_rows(d):
    """Bounds of the rows of a part, from the workspace: it holds 2 rows / part slots of K * C sums."""
    slots = cb.cbw_expert_workspace_size(d) // (4 * d.C * d.K)
    assert slots > 0
    return 2 * d.rows // (slots + 1) + 1, 2 * d.rows // slots


def _around(E, lengths):
    """Offsets of E experts of which only `lengths` (expert: rows) have rows."""
    off = [0]
    for e in range(E):
        off.append(off[-1] + lengths.get(e, 0))
    return off


# (rows, C, K, the experts' lengths, number of experts).  The part length
# follows from the capacity `rows`, which the lengths need not fill.
SPLIT = [
    (9300, 72, 40, {0: 4000, 2: 1, 3: 3299, 4: 600, 5: 1400}, 6),
    (9300, 72, 40, {0: 3299, 1: 400, 3: 517, 5: 1}, 6),
    # split experts on both sides of the 64th, whole ones between them
    (108000, 24, 16, {**{e: 3 * e + 1 for e in range(5, 70, 2)}, 2: 1500, 62: 700, 63: 514, 64: 5000, 66: 1025, 69: 600}, 70),
    # tiles of 256 x 256 (bf16)
    (16400, 520, 520, {**{e: 4 * e for e in range(4, 40)}, 0: 3000, 41: 1026, 50: 2049, 63: 1023}, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C,K,lengths,E", SPLIT, ids=lambda v: str(v) if isinstance(v, int) else "")
def test_parts_of_several_experts(rows, C, K, lengths, E, dtype):
    """At least two experts are taken in parts and at least one is not, twice
    over a workspace that held other sums: within the bound, and the same bits."""
    print("[case]", dtype, rows, C, K, E, flush=True)
    off = _around(E, lengths)
    assert off[-1] <= rows
    d = cb.ExpertDesc.make(E, rows, C, K, dtype)
    lo, hi = _part_rows(d)
    assert sum(n > hi for n in lengths.values()) >= 2 and any(0 < n <= lo for n in lengths.values())
    x, _, dy, _ = _draw(off, rows, C, K, dtype, 11)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    got = []
    for fill in (0, 255):
        ws = torch.full((cb.cbw_expert_workspace_size(d),), fill, dtype=torch.uint8, device="cuda")
        dW = torch.full((E, K, C), float("nan"), device="cuda")
        cb.expert_bwd_weight(d, x.cuda(), dy.cuda(), o, dW, ws)
        got.append(dW)
    assert torch.equal(*got)
    ref.check(got[0], *ref.expert_bwd_weight(x, dy, off), "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C,K", [(40, 64, 64), (700, 128, 1056)])
def test_relu_of_nonfinite_sums(rows, C, K, dtype):
    """ReLU gives +0.0 for a NaN sum and for -infinity, and marks both dead;
    +infinity stays and is live."""
    off = [0, rows // 3, rows]
    x, w, _, _ = _draw(off, rows, C, K, dtype, 12)
    w[:, :, 0] = torch.where(torch.arange(K) % 2 == 0, 1.0, -1.0).to(w.dtype)
    x[5, 0], x[rows - 1, 0], x[rows // 2, 1] = float("inf"), -float("inf"), float("nan")
    d = cb.ExpertDesc.make(2, rows, C, K, dtype)
    Y = torch.full((rows, K), -1.0, dtype=DT[dtype], device="cuda")
    mask = torch.zeros((rows * K + 31) // 32, dtype=torch.int32, device="cuda")
    cb.expert_fwd(d, x.cuda(), w.cuda(), torch.tensor(off, dtype=torch.int32, device="cuda"), Y, mask, cb.expert_workspace(d),
                  cb.CBW_FLAG_RELU)
    y = Y.cpu()
    bits = y.view(torch.int16 if dtype == "bf16" else torch.int32)
    assert torch.equal(y[5, 0::2], torch.full((K // 2,), float("inf"), dtype=y.dtype)) and (bits[5, 1::2] == 0).all()
    assert torch.equal(y[-1, 1::2], torch.full((K // 2,), float("inf"), dtype=y.dtype)) and (bits[-1, 0::2] == 0).all()
    assert (bits[rows // 2] == 0).all() and not y.isnan().any()
    assert torch.equal(mask.cpu(), ref.bits(y > 0))
