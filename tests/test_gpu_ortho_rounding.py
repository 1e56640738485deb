"""Five Newton-Schulz steps where singular values are far from alike: few live rows
(dead channels, experts that saw few tokens), few directions, single entries.  The
arithmetic of a bf16 result is that of a float32 one, and one rounding."""
import pytest
import torch

import ortho_gain
import ortho_ref as ref
import paper_2109_07710_amd as cb
from test_gpu_ortho import CUBIC, QUINTIC, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


def _draw(kind, live, batch, rows, cols, seed=5):
    """rows, columns: `live` of them hold values; rank: `live` directions (and noise of 1e-4 of them); strong: `live` strong
    rows above noise of 1e-4; diagonal: a value each in `live` rows; quarter: as gradients of a whole layer."""
    g = torch.Generator().manual_seed(seed)
    new = lambda *n: torch.randn(n, generator=g)  # noqa: E731
    out = torch.zeros(batch, rows, cols)
    for m in out:
        at = torch.randperm(cols if kind == "columns" else rows, generator=g)[:live]
        if kind == "rows":
            m[at] = new(live, cols)
        elif kind == "columns":
            m[:, at] = new(rows, live)
        elif kind == "strong":
            m.copy_(1e-4 * new(rows, cols))
            m[at] = new(live, cols)
        elif kind == "diagonal":
            m[at, at % cols] = 0.1 + new(live).abs()
        elif kind == "rank":
            m.copy_(new(rows, live) @ new(live, cols) + 1e-4 * new(rows, cols))
        else:
            m.copy_(new(rows, live) @ new(live, cols) / live ** 0.5 + 0.3 * new(rows, cols))
    return out


CASES = [("rows", 1, 1, 300, 700), ("rows", 4, 1, 128, 512), ("rows", 4, 2, 512, 512), ("rows", 32, 1, 1024, 1024), ("rows", 4, 1, 2048, 2048),
         ("columns", 4, 1, 700, 300), ("columns", 5, 1, 300, 700), ("strong", 4, 1, 260, 400), ("diagonal", 130, 2, 260, 400), ("rank", 4, 1, 300, 500),
         ("rows", 4, 14, 1100, 1200), ("columns", 4, 14, 1200, 1100), ("rows", 3, 70, 130, 200),
         ("quarter", 96, 1, 384, 640), ("quarter", 33, 2, 130, 260), ("rows", 5, 3, 64, 576), ("rows", 3, 2, 40, 100), ("rows", 2, 1, 3000, 20)]
_name = lambda c: "%s%d_%dx%dx%d" % c  # noqa: E731


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_bf16_result_is_the_float32_one_rounded(case):
    """Bit for bit: the products and X take the same bits whatever type the result has."""
    print("[case]", case, flush=True)
    m = _draw(*case)
    for steps, co in ((5, QUINTIC), (3, QUINTIC), (4, CUBIC)):
        assert torch.equal(_run(m, "bf16", "f32", co, steps), _run(m, "f32", "f32", co, steps).to(torch.bfloat16)), (steps, co)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] not in ("rank", "strong")], ids=_name)
def test_five_steps_of_unlike_singular_values(case):
    """Against 64 bits, with a bound below the rounding of a bf16 result; rows and columns of zeros stay zeros exactly."""
    print("[case]", case, flush=True)
    m = _draw(*case)
    o32, o16 = _run(m).cpu().double(), _run(m, "bf16").cpu().double()
    for i in range(min(case[2], 3)):
        r, c = m[i].abs().amax(1) > 0, m[i].abs().amax(0) > 0
        block = m[i][r][:, c]
        # (the block's own shape may be tall where the matrix is not: p(X) is the same from both sides)
        want = torch.zeros_like(o32[i])
        want[torch.nonzero(r), torch.nonzero(c).flatten()] = ref.steps_of(block, QUINTIC, 5, 1e-7, [True] * 5)[0]
        size, bound = float(want.norm()), ortho_gain.bound_of(m[i], QUINTIC, 5, 1e-7)
        assert bound <= 2.0 ** -8 * size, "no bound"
        for got, rounding in ((o32[i], 0.0), (o16[i], 2.0 ** -8)):
            assert bool((got[~r] == 0).all()) and bool((got[:, ~c] == 0).all())
            off = float((got - want).norm())
            assert off <= bound + rounding * size, "off by %.3g, %.3g allowed, of %.3g" % (off, bound + rounding * size, size)
