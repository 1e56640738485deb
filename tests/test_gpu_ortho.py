"""Orthogonalised updates against 64 bits: sizes that fill no tile, wide and
tall, batches, strides, all types, matrices of zeros and of no numbers."""
import pytest
import torch

import ortho_ref as ref
import paper_2109_07710_amd as cb

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _draw(batch, rows, cols, seed, rank=0.25):
    g = torch.Generator().manual_seed(seed)
    r = max(1, int(min(rows, cols) * rank))
    m = torch.randn((batch, rows, r), generator=g) @ torch.randn((batch, r, cols), generator=g) / r ** 0.5
    return (m + 0.3 * torch.randn((batch, rows, cols), generator=g)) * torch.logspace(-3, 1, batch)[:, None, None]


def _workspace(d):
    ws = cb.ortho_workspace(d)
    return ws.fill_(0xff)                   # (NaN in every type: nothing is read before it is written)


def _run(m, out="f32", dtype="f32", coefficients=QUINTIC, steps=5, eps=1e-7):
    batch, rows, cols = m.shape
    d = cb.OrthoDesc.make(rows, cols, batch, dtype, out, steps, coefficients, eps)
    o = torch.full((batch, rows, cols), float("nan"), dtype=DT[out], device="cuda")
    cb.grad_orthogonalize(d, m.to(DT[dtype]).cuda(), o, _workspace(d))
    return o


SIZES = [(1, 1, 1), (2, 1, 7), (2, 7, 1), (3, 5, 3), (2, 3, 40), (1, 1, 5000), (1, 4100, 2), (2, 64, 64), (1, 63, 65), (1, 64, 576),
         (2, 200, 104), (1, 129, 300), (3, 300, 129), (1, 257, 260), (2, 333, 257), (1, 513, 100), (1, 100, 2000), (1, 384, 640), (1, 300, 1500),
         (2, 16, 2048), (1, 2049, 16), (1, 13, 50000), (2, 17, 500), (1, 600, 32), (1, 20, 9000), (2, 33, 128), (1, 64, 129), (1, 50, 6100),
         (1, 40, 6200), (70, 9, 30), (3, 65, 64)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%dx%d" % s)
def test_steps(size, out):
    print("[case]", size, out, flush=True)
    m = _draw(*size, 1)
    dtype = "bf16" if size[1] % 2 else "f32"
    m = m.to(DT[dtype]).float()
    for steps, co in ((1, QUINTIC), (2, CUBIC), (5, QUINTIC)):
        o = _run(m, out, dtype, co, steps)
        for i in range(size[0]):
            ref.check(o[i], m[i], co, steps, 1e-7, "%s matrix %d, %d steps" % (size, i, steps))
    assert torch.equal(o, _run(m, out, dtype)), "the same call, the same bits"


def test_slow_coefficients():
    """A first coefficient below 1, with one large singular value: its steps are B X for the most part, and take both parts."""
    m = _draw(1, 200, 300, 8)[0]
    u, v = torch.linalg.qr(torch.randn((200, 1), generator=torch.Generator().manual_seed(3)))[0], torch.randn((1, 300), generator=torch.Generator().manual_seed(4))
    m = 0.01 * m / m.norm() + u @ (v / v.norm())
    for out in ("f32", "bf16"):
        ref.check(_run(m[None], out, coefficients=(0.25, 1.0, -0.25))[0], m, (0.25, 1.0, -0.25), 5, 1e-7, out)


def test_large():
    m = _draw(1, 700, 1600, 2)
    for out in ("f32", "bf16"):
        ref.check(_run(m, out)[0], m[0], QUINTIC, 5, 1e-7, out)
        ref.check(_run(m.transpose(1, 2).contiguous(), out)[0], m[0].t(), QUINTIC, 5, 1e-7, out + " tall")


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,cols", [(44, 640, 900), (44, 1100, 600), (70, 300, 300), (86, 260, 270)])
def test_large_batch(batch, rows, cols, out):
    """Enough for tiles of 256 on both sides of a whole turn, the last ones half empty; one matrix of zeros."""
    m = _draw(1, rows, cols, 7) * torch.linspace(0.5, 2.0, batch)[:, None, None]
    m[1::2] = m[1::2].flip(2)
    m[9] = 0.0
    o = _run(m, out)
    assert bool((o[9] == 0).all())
    for i in (0, 1, batch - 1):
        ref.check(o[i], m[i], QUINTIC, 5, 1e-7, "matrix %d" % i)
    # the others are the same matrices at other sizes, which the norm takes off but for eps and its rounding
    for i in range(2, batch):
        if i != 9:
            off = float((o[i].double() - o[i & 1].double()).norm() / o[i & 1].double().norm())
            assert off <= (2.0 ** -7 if out == "bf16" else 2.0 ** -16), (i, off)
    assert torch.equal(o, _run(m, out)), "the same call, the same bits"


def test_becomes_orthogonal():
    """Cubic steps converge: X X^T = I to the last step's own error.  Its products, 96 long, are off by 8e-7 an entry (R is below
    0.1) and dA by 2e-6 more on the diagonal (see ortho_ref); dA enters X X^T once, d(B X) twice through a row of 96 values:
    2.8e-6 + 2 sqrt(96) 4e-7 < 2^-16."""
    q = torch.linalg.qr(torch.randn((96, 96), generator=torch.Generator().manual_seed(1)))[0]
    m = (q * torch.linspace(0.2, 1.0, 96)) @ torch.randn((96, 96), generator=torch.Generator().manual_seed(2)).double().float()
    m = q @ torch.diag(torch.linspace(0.2, 1.0, 96)) @ torch.linalg.qr(m)[0]
    o = _run(m[None], coefficients=CUBIC, steps=20)[0].cpu().double()
    assert float((o @ o.t() - torch.eye(96, dtype=torch.float64)).abs().max()) <= 2.0 ** -16


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,cols", [(70, 33), (33, 70), (130, 260)])
def test_strides_and_alignment(rows, cols, dtype, out):
    """Rows apart, with NaN between them, at addresses of one element's alignment; what lies between O's rows stays."""
    batch, si, so = 2, cols + 5, cols + 3
    m = _draw(batch, rows, cols, 3).to(DT[dtype])
    src = torch.full((1 + batch * rows * si,), float("nan"), dtype=DT[dtype], device="cuda")
    dst = torch.full((1 + batch * rows * so,), 7.0, dtype=DT[out], device="cuda")
    M = src[1:].view(batch, rows, si)[:, :, :cols]
    O = dst[1:].view(batch, rows, so)[:, :, :cols]
    M.copy_(m)
    d = cb.OrthoDesc.make(rows, cols, batch, dtype, out, in_stride=si, out_stride=so)
    cb.grad_orthogonalize(d, M, O, _workspace(d))
    assert torch.equal(O, _run(m.float(), out, dtype))
    assert bool((dst[1:].view(batch, rows, so)[:, :, cols:] == 7).all()) and float(dst[0]) == 7.0


def test_in_place_and_filter_shapes():
    m = _draw(1, 32, 72, 4)[0]
    want = _run(m[None])[0]
    d = cb.OrthoDesc.make(32, 72)
    f = m.view(32, 3, 3, 8).cuda()                                   # a convolution's filter, [K][R][S][C]
    cb.grad_orthogonalize(d, f, f, _workspace(d))
    assert torch.equal(f.view(32, 72), want)


@pytest.mark.parametrize("rows,cols", [(40, 24), (20, 300), (200, 300)])
def test_zeros_and_no_numbers(rows, cols):
    """A matrix of zeros gives zeros, one with a NaN or an infinity NaN throughout; the others of the batch are as alone."""
    m = _draw(5, rows, cols, 5)
    m[1] = 0.0
    m[2, rows // 2, cols // 3] = float("nan")
    m[3, 0, cols - 1] = float("-inf")
    for out in ("f32", "bf16"):
        o = _run(m, out)
        assert bool((o[1] == 0).all()) and bool(torch.isnan(o[2]).all()) and bool(torch.isnan(o[3]).all())
        for i in (0, 4):
            ref.check(o[i], m[i], QUINTIC, 5, 1e-7, "matrix %d" % i)
        clean = m.clone()
        clean[1:4] = 1.0
        assert torch.equal(o[[0, 4]], _run(clean, out)[[0, 4]])
    assert bool((_run(m[1:2], eps=0.0) == 0).all())


@pytest.mark.parametrize("size", [1e-37, 1e-30, 1e-7, 1e18, 1e30])
def test_sizes_of_values(size):
    """The norm is taken in 64 bits: squares of no size overflow or vanish.  eps counts where it is as large as the norm."""
    m = _draw(1, 48, 100, 6) / 10
    m = (m / m.norm() * size).float()
    eps = 0.0 if size < 1e-7 else 1e-7
    ref.check(_run(m, eps=eps)[0], m[0], QUINTIC, 5, eps, "%g" % size)


@pytest.mark.parametrize("first,second", [((2, 96, 200), (1, 300, 260)), ((3, 64, 576), (70, 260, 300)), ((9, 16, 40), (2, 2000, 30))],
                         ids=["general", "panels_large", "whole_tall"])
def test_captured(first, second):
    """In a graph with another call over its own workspace, replayed with other inputs between eager calls."""
    da, db = cb.OrthoDesc.make(*first[1:], first[0]), cb.OrthoDesc.make(*second[1:], second[0], "f32", "bf16")
    sets = [(_draw(*first, s).cuda(), _draw(*second, s + 9).cuda()) for s in range(3)]
    a, b = (t.clone() for t in sets[0])
    oa, ob = torch.empty_like(a), torch.empty(b.shape, dtype=torch.bfloat16, device="cuda")
    wa, wb, we = _workspace(da), _workspace(db), torch.empty(max(_workspace(da).numel(), _workspace(db).numel()), dtype=torch.uint8, device="cuda")

    def step(x, y, ws_a, ws_b):
        cb.grad_orthogonalize(da, a, x, ws_a)
        cb.grad_orthogonalize(db, b, y, ws_b)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(oa, ob, wa, wb)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(oa, ob, wa, wb)
    for k in (1, 2, 0, 1):
        a.copy_(sets[k][0]), b.copy_(sets[k][1])
        oa.zero_(), ob.zero_()
        graph.replay()
        ea, eb = torch.zeros_like(oa), torch.zeros_like(ob)
        step(ea, eb, we, we)
        torch.cuda.synchronize()
        assert torch.equal(oa, ea) and torch.equal(ob, eb)


@pytest.mark.parametrize("rows,cols", [(3, 1 << 20), ((1 << 20) - 1, 2)])
def test_longest(rows, cols):
    m = _draw(1, rows, cols, 9)
    co = QUINTIC if rows < cols else CUBIC
    ref.check(_run(m, coefficients=co)[0], m[0], co, 5, 1e-7, "longest")


def test_one_large_matrix():
    """5120 x 5120, ten times the same block on its diagonal: every block as alone beside a norm sqrt(10) as large, the rest zero."""
    n, blocks = 512, 10
    m = _draw(1, n, n, 13)[0]
    M = torch.block_diag(*[m] * blocks)
    o = _run(M[None])[0]
    eps = (blocks ** 0.5 - 1.0) * float(m.double().norm())
    for i in range(blocks):
        ref.check(o[i * n:(i + 1) * n, i * n:(i + 1) * n], m, QUINTIC, 5, eps, "block %d" % i)
        o[i * n:(i + 1) * n, i * n:(i + 1) * n] = 0.0
    assert not bool(o.any())


def test_rows_past_32_bits():
    """Rows so far apart that their addresses pass 2^32 elements, in M and in O."""
    rows, cols, stride = 2100, 40, 1 << 21
    m = _draw(1, rows, cols, 10)[0]
    M = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)[:, :cols]
    O = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)[:, :cols]
    M.copy_(m.to(torch.bfloat16))
    d = cb.OrthoDesc.make(rows, cols, 1, "bf16", "bf16", in_stride=stride, out_stride=stride)
    cb.grad_orthogonalize(d, M, O, _workspace(d))
    assert torch.equal(O, _run(m.to(torch.bfloat16).float()[None], "bf16", "bf16")[0])


def test_two_streams_at_once():
    """Calls of the same descriptor on two streams, each with its own workspace."""
    m = [_draw(4, 260, 300, s).cuda() for s in (11, 12)]
    d = cb.OrthoDesc.make(260, 300, 4)
    want = [_run(x) for x in m]
    streams, ws, out = [torch.cuda.Stream() for _ in m], [_workspace(d) for _ in m], [torch.zeros_like(x) for x in m]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, x, w, o in zip(streams, m, ws, out):
            cb.grad_orthogonalize(d, x, o, w, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(out, want))


def test_update_of_an_expert_layer():
    """From a gated layer's rows to its update: gradients by expert, one expert without rows, orthogonalised in place."""
    off, rows, C, K = [0, 40, 40, 200], 200, 64, 96
    E = len(off) - 1
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = torch.randn((rows, C), generator=g, device="cuda"), torch.randn((rows, C), generator=g, device="cuda")
    w, w2 = torch.randn((E, 2, K, C), generator=g, device="cuda") / 8, torch.randn((E, C, K), generator=g, device="cuda") / 8
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    d = cb.GatedDesc.make(E, rows, C, K, "silu", "f32")
    H, GU, dW = torch.empty((rows, K), device="cuda"), torch.empty((rows, 2 * K), device="cuda"), torch.empty((E, 2 * K, C), device="cuda")
    cb.expert_gated_fwd(d, x, w, o, H, GU)
    cb.expert_gated_bwd(d, dy, w2, o, GU, GU)
    both = cb.ExpertDesc.make(E, rows, C, 2 * K, "f32")
    cb.expert_bwd_weight(both, x, GU, o, dW, cb.expert_workspace(both))
    grads = dW.cpu().view(2 * E, K, C)                                # a matrix for every filter, gate and up
    u = cb.OrthoDesc.make(K, C, 2 * E)
    cb.grad_orthogonalize(u, dW, dW, _workspace(u))
    got = dW.view(2 * E, K, C)
    assert bool((got[2:4] == 0).all())
    for i in (0, 1, 4, 5):
        ref.check(got[i], grads[i], QUINTIC, 5, 1e-7, "filter %d" % i)
