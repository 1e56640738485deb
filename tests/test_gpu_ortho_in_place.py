"""O in M's place, in every form of the orthogonalised update: bit for bit what a
result of its own holds."""
import pytest
import torch

import paper_2109_07710_amd as cb
from test_gpu_ortho import DT, _draw, _run, _workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cb.lib()


# one panel, wide and tall; several panels, wide and tall; tiles of 64, wide and
# tall; of 128; of 256 and their quarters; more matrices than lanes
SIZES = [(3, 40, 24), (3, 20, 100), (3, 64, 576), (2, 3000, 50), (3, 200, 300), (3, 300, 200), (2, 1500, 1600), (15, 1100, 1200), (15, 1200, 1100),
         (70, 130, 70)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%dx%d" % s)
def test_in_place(size, dtype):
    """Adjacent, and with rows apart by as much in both and something else between them; one matrix of zeros among them."""
    print("[case]", size, dtype, flush=True)
    batch, rows, cols = size
    m = _draw(batch, rows, cols, 21)
    m[1] = 0.0
    want = _run(m, dtype, dtype)
    assert bool((want[1] == 0).all()) and bool(torch.isfinite(want).all())
    d = cb.OrthoDesc.make(rows, cols, batch, dtype, dtype)
    x = m.to(DT[dtype]).cuda()
    cb.grad_orthogonalize(d, x, x, _workspace(d))
    assert torch.equal(x, want)
    stride = cols + 3
    d = cb.OrthoDesc.make(rows, cols, batch, dtype, dtype, in_stride=stride, out_stride=stride)
    space = torch.full((batch, rows, stride), float("nan"), dtype=DT[dtype], device="cuda")
    x = space[:, :, :cols]
    x.copy_(m)
    cb.grad_orthogonalize(d, x, x, _workspace(d))
    assert torch.equal(x, want) and bool(torch.isnan(space[:, :, cols:]).all())
