"""Which shapes the orthogonalised update takes for a descriptor's matrices: on the
CPU with tensors that say they are a device's, and (marked) through the call."""
import pytest
import torch

import paper_2109_07710_amd as cb


class _OnDevice(torch.Tensor):
    is_cuda = True


def _take(d, *shape, stride=None):
    return cb._matrices(torch.zeros(shape).as_subclass(_OnDevice), d, d.cols if stride is None else stride, torch.float32)


@pytest.mark.parametrize("rows,cols,batch,shape", [
    (256, 2304, 1, (256, 2304)), (256, 2304, 1, (1, 256, 2304)), (32, 72, 1, (32, 3, 3, 8)), (32, 72, 2, (2, 32, 3, 3, 8)), (32, 72, 2, (64, 72)),
    (24, 16, 6, (3, 48, 16)),                       # [E][2K][C], a matrix for each of an expert's two filters
    (24, 16, 6, (3, 2, 24, 16)), (1, 40, 1, (40,)), (40, 1, 1, (40,)), (40, 1, 3, (3, 40)), (5, 7, 0, (0, 5, 7)), (5, 7, 0, (0,)), (6, 6, 2, (2, 6, 6)),
    (8, 24, 3, (24, 24, 1)), (40, 1, 1, (1, 40)), (1, 40, 1, (40, 1))])      # (a vector is the same matrix either way)
def test_shapes_that_are_the_matrices(rows, cols, batch, shape):
    _take(cb.OrthoDesc.make(rows, cols, batch), *shape)


@pytest.mark.parametrize("rows,cols,batch,shape", [
    (256, 2304, 1, (2304, 256)), (256, 2304, 1, (3, 3, 256, 256)), (8, 24, 3, (3, 24, 8)), (8, 24, 3, (3 * 8 * 24,)),
    (8, 24, 3, (2, 8, 24)), (32, 72, 1, (8, 3, 3, 32))])
def test_shapes_that_are_not(rows, cols, batch, shape):
    with pytest.raises(ValueError, match="expected"):
        _take(cb.OrthoDesc.make(rows, cols, batch), *shape)


def test_contiguous_is_still_asked_for():
    d = cb.OrthoDesc.make(8, 24)
    with pytest.raises(ValueError, match="contiguous"):
        cb._matrices(torch.zeros(24, 8).t().as_subclass(_OnDevice), d, 24, torch.float32)


@pytest.mark.gpu
def test_call_refuses_the_other_shape():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    d = cb.OrthoDesc.make(72, 200)
    m, ws = torch.ones(72, 200, device="cuda"), cb.ortho_workspace(d)
    for a, b in ((m.view(200, 72), m), (m, m.view(200, 72))):
        with pytest.raises(ValueError, match="expected"):
            cb.grad_orthogonalize(d, a, b, ws)
