"""Host-only checks of the gated layer's operators: descriptors and every
refusal that comes before a launch."""
import ctypes

import pytest
import torch

import paper_2109_07710_amd as cb

FAKE, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 4)
INV, UNS = cb.CBW_ERR_INVALID_ARG, cb.CBW_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(cb.LIB_PATH):
        pytest.skip("library not built")
    return cb.lib()


def _desc(**kw):
    a = dict(E=4, rows=100, C=64, K=32)
    a.update(kw)
    return cb.GatedDesc.make(**a)


def test_descriptors(L):
    ok = cb.cbw_validate_gated_desc
    assert ok(_desc()) == ok(_desc(rows=0)) == ok(_desc(E=1024)) == ok(_desc(act="gelu")) == cb.CBW_OK
    assert ok(_desc(x_stride=72, h_stride=40, gu_stride=72)) == ok(_desc(C=12, K=4, dtype="f32")) == cb.CBW_OK
    for bad in (dict(E=0), dict(rows=-1), dict(C=0), dict(K=-8), dict(K=0), dict(x_stride=56), dict(h_stride=24), dict(gu_stride=56)):
        assert ok(_desc(**bad)) == INV, bad
    for bad in (dict(C=12), dict(K=4), dict(x_stride=68), dict(h_stride=36), dict(gu_stride=68), dict(E=1025), dict(rows=1 << 31),
                dict(x_stride=1 << 20), dict(gu_stride=1 << 20), dict(C=32768, K=8192), dict(C=6, dtype="f32"), dict(K=1 << 30)):
        assert ok(_desc(**bad)) == UNS, bad
    for field, value in (("dtype", 5), ("act", 4), ("act", -1), ("reserved", 1)):
        d = _desc()
        setattr(d, field, value)
        assert ok(d) == INV, field
    assert L.cbw_validate_gated_desc(None) == INV


def test_refusals(L):
    def fwd(d=None, X=FAKE, W=FAKE, o=FAKE, H=FAKE, GU=FAKE):
        return L.expert_gated_fwd(ctypes.byref(d or _desc()), X, W, o, H, GU, None)

    def bwd(d=None, dY=FAKE, W2=FAKE, o=FAKE, GU=FAKE, dGU=FAKE, H=FAKE):
        return L.expert_gated_bwd(ctypes.byref(d or _desc()), dY, W2, o, GU, dGU, H, None)

    for call, names in ((fwd, ("X", "W", "o", "H")), (bwd, ("dY", "W2", "o", "GU", "dGU"))):
        for n in names:
            assert call(**{n: None}) == INV, n
        for n in names + (("GU",) if call is fwd else ("H",)):
            assert call(**{n: ctypes.c_void_p((1 << 20) + 2)}) == UNS, n
            assert n == "o" or call(**{n: ODD}) == UNS, n
        assert call(d=_desc(K=12)) == UNS and call(d=_desc(E=0)) == INV
    none = dict.fromkeys(("X", "W", "H", "GU"))
    assert fwd(d=_desc(rows=0), **none) == cb.CBW_OK
    assert bwd(d=_desc(rows=0), **dict.fromkeys(("dY", "W2", "GU", "dGU", "H"))) == cb.CBW_OK
    assert L.expert_gated_fwd(None, FAKE, FAKE, FAKE, FAKE, FAKE, None) == INV
    assert L.expert_gated_bwd(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == INV


def test_binding_refuses_host_tensors():
    d = _desc()
    x, w, h = torch.zeros(100, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 32, 64, dtype=torch.bfloat16), torch.zeros(100, 32, dtype=torch.bfloat16)
    o = torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        cb.expert_gated_fwd(d, x, w, o, h)
    with pytest.raises(ValueError, match="device"):
        cb.expert_gated_bwd(d, x, torch.zeros(4, 64, 32, dtype=torch.bfloat16), o, torch.zeros(100, 64, dtype=torch.bfloat16),
                            torch.zeros(100, 64, dtype=torch.bfloat16))
