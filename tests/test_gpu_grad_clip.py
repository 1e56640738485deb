"""The norm of many gradients and their clipping, against 64 bits."""
import math

import pytest
import torch

import block_ref as ref
import paper_2109_07710_amd as cb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _exact(grads, kind):
    v = torch.cat([g.detach().cpu().double().flatten() for g in grads] + [torch.zeros(1, dtype=torch.float64)])
    return float(v.square().sum().sqrt() if kind == "2" else v.abs().max())


def _check(grads, max_norm, kind="2", in_place=False, outs=None):
    before = [g.detach().cpu().double() for g in grads]
    want = _exact(grads, kind)
    outs = grads if in_place else [torch.full_like(g, 7.0) for g in grads] if outs is None else outs
    lst = cb.GradList(grads, None if in_place else outs)
    ws = cb.grad_workspace(lst)
    ws.fill_(255)
    only = torch.full((1,), 7.0, device="cuda")
    cb.grad_norm(lst, only, ws, kind)
    norm = torch.full((2,), 7.0, device="cuda")
    cb.grad_clip(lst, max_norm, norm, ws, kind)
    # a 64-bit sum, rounded once; c one more rounding
    got, c = (float(v) for v in norm)
    assert abs(got - want) <= 1.01 * ref.U32 * want and got == float(only)
    c_want = min(1.0, max_norm / (want + 1e-6))
    assert abs(c - c_want) <= 2 * ref.U32 * c_want and (c_want < 1 or c == 1.0)
    for b, g, o in zip(before, grads, outs):
        # c, the product and the rounding to the type
        ref.check(o, b * c_want, 4 * ref.U32 * (b * c_want).abs(), "out")
        if not in_place:
            assert torch.equal(g.detach().cpu().double(), b), "a gradient was written"
    return norm


def _draw(sizes, types, seed=1, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(torch.bfloat16 if t else torch.float32).cuda()
            for n, t in zip(sizes, types)]


SIZES = [[1], [7], [8], [9], [8191, 8192, 8193], [3, 1, 4, 1, 5, 9, 2, 6], [100000, 1, 33], [1] * 129, [5] * 300,
         [64, 0, 3, 0, 0, 20000, 0]]


@pytest.mark.parametrize("kind", ["2", "inf"])
@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "n%d_%d" % (len(s), sum(s)))
def test_sizes(sizes, types, kind):
    t = [types == "bf16" or types == "mixed" and i % 2 for i in range(len(sizes))]
    for max_norm, in_place in ((2.0 ** -7, False), (0.5, True), (2.0 ** 30, False), (2.0 ** 30, True)):
        _check(_draw(sizes, t), max_norm, kind, in_place)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_views(dtype):
    """Gradients and outputs that are views into packed buffers, at every
    alignment of their elements; nothing between or beside them is written."""
    n = [3, 16, 17, 8200, 1, 31, 4096]
    flat = torch.randn(sum(n) + 40, device="cuda").to(dtype)
    out = torch.full((sum(n) + 40,), 9.0, dtype=dtype, device="cuda")
    grads, outs, at = [], [], 5
    for i, k in enumerate(n):
        grads.append(flat[at:at + k])
        outs.append(out[at + 2:at + 2 + k])
        at += k + 3
    _check(grads, 0.25, outs=outs)
    mask = torch.ones(out.numel(), dtype=torch.bool)
    for o in outs:
        mask[o.storage_offset():o.storage_offset() + o.numel()] = False
    assert (out.cpu()[mask] == 9).all()


def test_many_chunks():
    """More chunks than workgroups, in one tensor and beside small ones."""
    _check(_draw([5, 30000001, 7, 4000003], [0, 0, 1, 1]), 1.0)


def test_large_and_small_values():
    """Squares beyond float32's range, and below it, in float32 and bf16."""
    for t in (0, 1):
        _check(_draw([1000, 5000], [t, t], scale=1e25), 1.0)
        _check(_draw([1000, 5000], [t, t], scale=1e-25), 1.0)
    g = _draw([4096], [0])
    g[0].fill_(3e38)
    lst = cb.GradList(g)
    norm, ws = torch.zeros(2, device="cuda"), cb.grad_workspace(lst)
    cb.grad_norm(lst, norm, ws)
    assert math.isinf(float(norm[0]))       # 64 * 3e38 is past float32


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["2", "inf"])
def test_nonfinite(kind, dtype):
    """Infinity: c = 0, finite values become zeros and the infinite one NaN.
    NaN anywhere: the norm, c and all values are NaN."""
    for bad in (float("inf"), -float("inf"), float("nan")):
        g = [torch.ones(5000, device="cuda").to(dtype) for _ in range(3)]
        g[1][4321] = bad
        lst = cb.GradList(g)
        norm, ws = torch.zeros(2, device="cuda"), cb.grad_workspace(lst)
        cb.grad_clip(lst, 1.0, norm, ws, kind)
        if math.isnan(bad):
            assert torch.isnan(norm).all() and all(torch.isnan(v).all() for v in g)
        else:
            assert float(norm[0]) == math.inf and float(norm[1]) == 0.0
            assert (g[0] == 0).all() and torch.isnan(g[1][4321]) and (g[1][:4321] == 0).all()


def test_no_tensors():
    for grads in ([], [torch.empty(0, device="cuda")]):
        lst = cb.GradList(grads)
        norm, ws = torch.full((2,), 7.0, device="cuda"), cb.grad_workspace(lst)
        cb.grad_clip(lst, 1.0, norm, ws)
        assert norm.tolist() == [0.0, 1.0]
        cb.grad_norm(lst, norm, ws, "inf")
        assert float(norm[0]) == 0.0


def test_limits():
    """max_norm 0: everything becomes zero; infinity: nothing changes."""
    g = _draw([1000], [0])
    assert _check(g, 0.0).tolist()[1] == 0.0
    lst = cb.GradList(g)
    before, norm, ws = g[0].clone(), torch.zeros(2, device="cuda"), cb.grad_workspace(lst)
    cb.grad_clip(lst, math.inf, norm, ws)
    assert torch.equal(g[0], before) and float(norm[1]) == 1.0


def test_graph_with_many_tensors():
    """Captured (the addresses travel in the launches): every replay clips
    what the gradients hold then."""
    g = _draw([100 + i for i in range(300)], [i % 3 == 0 for i in range(300)])
    outs = [torch.zeros_like(v) for v in g]
    lst = cb.GradList(g, outs)
    ws, norm = cb.grad_workspace(lst), torch.zeros(2, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    cb.grad_clip(lst, 1.0, norm, ws, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cb.grad_clip(lst, 1.0, norm, ws, stream=torch.cuda.current_stream())
    for k in range(4):
        g[k].mul_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        want = _exact(g, "2")
        assert abs(float(norm[0]) - want) <= 1.01 * ref.U32 * want
        for a, o in zip(g, outs):
            b = a.cpu().double() / (want + 1e-6)
            ref.check(o, b, 4 * ref.U32 * b.abs(), "out")


def test_binding_refuses():
    a = torch.zeros(8, device="cuda")
    for g, o in (([a.half()], None), ([a], [a, a]), ([a], [a[:4]]), ([a], [a.bfloat16()]), ([a[::2]], None),
                 ([torch.zeros(8)], None)):
        with pytest.raises(ValueError):
            cb.GradList(g, o)
    lst = cb.GradList([a])
    norm, ws = torch.zeros(2, device="cuda"), cb.grad_workspace(lst)
    for bad in (-1.0, math.nan):
        with pytest.raises(cb.CbwError):
            cb.grad_clip(lst, bad, norm, ws)
    with pytest.raises(ValueError):
        cb.grad_clip(lst, 1.0, norm[:1], ws)
    with pytest.raises(cb.CbwError) as e:
        cb.grad_clip(lst, 1.0, norm, ws[:8])
    assert e.value.status == cb.CBW_ERR_WORKSPACE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1.0, 1e10, 3e38, math.inf])
def test_norm_past_float32(dtype, max_norm):
    """Finite gradients whose 2-norm no float32 holds: the norm is infinity and
    c is 0, as for an infinite gradient, whatever the limit is."""
    g = [torch.full((n,), 3e38, device="cuda").to(dtype) for n in (4096, 5)]
    lst = cb.GradList(g, [torch.full_like(v, 7.0) for v in g])
    norm, ws = torch.full((2,), 7.0, device="cuda"), cb.grad_workspace(lst)
    cb.grad_clip(lst, max_norm, norm, ws)
    assert norm.tolist() == [math.inf, 0.0]
    assert all((o == 0).all() for o in lst.outs)
    # and the largest magnitude, which float32 holds, is a norm like any other
    cb.grad_clip(lst, 1.0, norm, ws, "inf")
    assert 0 < float(norm[1]) and float(norm[0]) == float(g[0][0])


@pytest.mark.parametrize("kind", ["2", "inf"])
def test_infinite_norm_without_a_limit(kind):
    """An infinite gradient gives c = 0 where the limit is infinite as well."""
    g = [torch.ones(3000, device="cuda") for _ in range(2)]
    g[1][7] = -math.inf
    lst = cb.GradList(g)
    norm, ws = torch.full((2,), 7.0, device="cuda"), cb.grad_workspace(lst)
    cb.grad_clip(lst, math.inf, norm, ws, kind)
    assert norm.tolist() == [math.inf, 0.0]
    assert (g[0] == 0).all() and torch.isnan(g[1][7]) and (g[1][8:] == 0).all()
