"""Host-only checks of the orthogonalised update: descriptors, the coefficients
that are let through, workspace sizes, and every refusal before a launch."""
import ctypes

import pytest
import torch

import paper_2109_07710_amd as cb

FAKE, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 4)
INV, UNS, WSP = cb.CBW_ERR_INVALID_ARG, cb.CBW_ERR_UNSUPPORTED, cb.CBW_ERR_WORKSPACE


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(cb.LIB_PATH):
        pytest.skip("library not built")
    return cb.lib()


def _desc(**kw):
    a = dict(rows=100, cols=64, batch=2)
    a.update(kw)
    return cb.OrthoDesc.make(**a)


def test_descriptors(L):
    ok = cb.cbw_validate_ortho_desc
    assert ok(_desc()) == ok(_desc(batch=0)) == ok(_desc(rows=1, cols=1)) == ok(_desc(rows=1 << 20, cols=3)) == cb.CBW_OK
    assert ok(_desc(rows=16384, cols=16384, batch=1)) == ok(_desc(eps=0.0)) == ok(_desc(in_stride=65, out_stride=99)) == cb.CBW_OK
    for bad in (dict(rows=0), dict(cols=-1), dict(batch=-1), dict(steps=0), dict(in_stride=63), dict(out_stride=0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(coefficients=(1.0, float("nan"), 0.0)),
                dict(coefficients=(float("inf"), 0.0, 0.0))):
        assert ok(_desc(**bad)) == INV, bad
    for bad in (dict(rows=(1 << 20) + 1), dict(rows=16385, cols=16385), dict(steps=101), dict(in_stride=(1 << 31) + 1),
                dict(batch=1 << 22), dict(rows=16384, cols=16384, batch=70)):
        assert ok(_desc(**bad)) == UNS, bad
    for field in ("dtype", "out_dtype"):
        d = _desc()
        setattr(d, field, 3)
        assert ok(d) == INV, field
    assert L.cbw_validate_ortho_desc(None) == INV


def _grows(coefficients, steps):
    """Largest |p(v)| and |b l + c l^2| on the way from [0, 1], by a fine grid."""
    a, b, c = (ctypes.c_float(v).value for v in coefficients)
    top, most, poly = 1.0, 0.0, 0.0
    for _ in range(steps):
        v = torch.linspace(0, top, 20001, dtype=torch.float64)
        poly = max(poly, float((v ** 2 * (b + c * v ** 2)).abs().max()))
        top = float((v * (a + v ** 2 * (b + v ** 2 * c))).abs().max())
        most = max(most, top)
        if most > 1e3:
            break
    return most, poly


@pytest.mark.parametrize("coefficients,steps", [
    ((3.4445, -4.7750, 2.0315), 5), ((3.4445, -4.7750, 2.0315), 100), ((1.5, -0.5, 0.0), 30), ((15 / 8, -10 / 8, 3 / 8), 20),
    ((4.5, -4.775, 2.0), 3), ((8.0, -20.0, 14.0), 4), ((3.0, 0.0, 0.0), 1), ((3.0, 0.0, 0.0), 2), ((5.0, -4.0, 0.0), 5), ((1.0, 1.0, 1.0), 3),
    ((0.0, 0.0, 0.0), 3), ((1.0, 40.0, -40.0), 1), ((0.0, 0.0, 3.0), 2), ((-2.0, 1.0, 0.0), 9), ((1.0, -40.0, 40.0), 1), ((2.0, -1.5, 0.5), 100)])
def test_coefficients(L, coefficients, steps):
    """Let through exactly where singular values stay below 4 and the polynomial's matrix below 32."""
    most, poly = _grows(coefficients, steps)
    want = cb.CBW_OK if most <= 4.0 and poly <= 32.0 else UNS
    assert cb.cbw_validate_ortho_desc(_desc(coefficients=coefficients, steps=steps)) == want, (most, poly)


def test_workspace(L):
    n = cb.cbw_ortho_workspace_size(_desc(rows=1024, cols=2048, batch=3))
    assert 3 * 1024 * 2048 * 12 <= n <= 3 * 1024 * 2048 * 12 + 3 * 1024 * 1024 * 8 + (1 << 26)
    assert cb.cbw_ortho_workspace_size(_desc(batch=0)) == cb.cbw_ortho_workspace_size(_desc()) == 0    # (one panel: all in the LDS)
    with pytest.raises(cb.CbwError):
        cb.cbw_ortho_workspace_size(_desc(rows=0))
    assert L.cbw_ortho_workspace_size(ctypes.byref(_desc()), None) == INV


def test_refusals(L):
    n = cb.cbw_ortho_workspace_size(_desc(rows=300, cols=200))
    assert n > 0

    def call(d=None, M=FAKE, O=ODD, ws=FAKE, nb=n):
        return L.grad_orthogonalize(ctypes.byref(d or _desc(rows=300, cols=200)), M, O, ws, nb, None)

    assert call(M=None) == call(O=None) == call(d=_desc(rows=0)) == INV
    assert call(O=FAKE, d=_desc(out_dtype="bf16")) == call(O=FAKE, d=_desc(out_stride=70)) == INV     # in place, not alike
    assert call(M=ctypes.c_void_p((1 << 20) + 2)) == call(O=ctypes.c_void_p((1 << 20) + 2)) == call(ws=ODD) == UNS
    assert call(d=_desc(dtype="bf16"), M=ctypes.c_void_p((1 << 20) + 1)) == call(d=_desc(steps=101)) == UNS
    assert call(ws=None) == call(nb=n - 1) == WSP
    assert call(d=_desc(batch=0), M=None, O=None, ws=None, nb=0) == cb.CBW_OK
    assert L.grad_orthogonalize(None, FAKE, ODD, FAKE, n, None) == INV


def test_binding_refuses_host_tensors():
    t = torch.zeros(2, 100, 64)
    with pytest.raises(ValueError, match="device"):
        cb.grad_orthogonalize(_desc(), t, t, torch.zeros(8, dtype=torch.uint8))
