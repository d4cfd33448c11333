"""Argument checks of the residual block's calls that need no GPU: every call below fails (or
has nothing to do) before any device call."""
import ctypes

import pytest
import torch

import paper_1909_11150_amd as fg

FAKE = 0x1000000          # never dereferenced
STEP = 0x1000000


@pytest.fixture(scope="module")
def L():
    return fg.lib()


def at(k):
    """Addresses far from each other."""
    return FAKE + k * STEP


def test_act8_sizes_and_refusals(L):
    assert fg.act8_bytes(3, 70) == 3 * 96 + 9 and fg.act8_bytes(0, 8) == 0
    assert fg.act8_bytes(1, 1) == 33
    for rows, cols in ((-1, 8), (4, 0), (1, 1 << 31), (1 << 30, 33), (1 << 29, 32)):
        assert fg.act8_bytes(rows, cols) == 0
    assert fg.act8_bytes((1 << 29) - 1, 32) == ((1 << 29) - 1) * 33
    for name in ("act8_pack", "act8_unpack"):
        fn = getattr(L, name)

        def call(x=at(0), p=at(1), none=False, **kw):
            d = fg.Act8Desc.make(**{**dict(rows=64, cols=40), **kw})
            a, b = (x, p) if name == "act8_pack" else (p, x)
            return fn(None if none else ctypes.byref(d), a, b, None)

        assert call(none=True) == fg.FG_EINVAL
        for bad in (dict(x=None), dict(p=None), dict(rows=-1), dict(cols=0), dict(dtype=3),
                    dict(x_ld=39), dict(x_ld=-40), dict(x=at(0) + 1), dict(p=at(1) + 8),
                    dict(x=at(0) + 2, dtype=fg.F32), dict(p=at(0) + 16), dict(p=at(0))):
            assert call(**bad) == fg.FG_EINVAL, bad
        for bad in (dict(rows=1 << 30), dict(rows=1, cols=1 << 31), dict(x_ld=1 << 58)):
            assert call(**bad) == fg.FG_EUNSUPPORTED, bad
        assert call(rows=0, x=None, p=None) == fg.FG_OK


def test_layer_norm_fwd_refusals(L):
    def call(none=False, x=at(0), w=at(1), b=at(2), y=at(3), stats=at(4), packed=at(5), **kw):
        d = fg.NormDesc.make(**{**dict(rows=64, cols=40), **kw})
        return L.layer_norm_fwd(None if none else ctypes.byref(d), x, w, b, y, stats, packed, None)

    assert call(none=True) == fg.FG_EINVAL
    for bad in (dict(x=None), dict(y=None), dict(rows=-1), dict(cols=0), dict(dtype=-1),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=1e-60),
                dict(eps=float("inf")), dict(x_ld=39), dict(y_ld=1), dict(add_ld=39),
                dict(dx_ld=-1), dict(x=at(0) + 1), dict(w=at(1) + 1), dict(stats=at(4) + 4),
                dict(packed=at(5) + 1), dict(y=at(0) + 2), dict(y=at(0), x_ld=48), dict(y=at(1)),
                dict(y=at(2)), dict(stats=at(0)), dict(packed=at(0)), dict(stats=at(3)),
                dict(packed=at(4)), dict(y=at(0) + 78, x_ld=96, y_ld=96)):
        assert call(**bad) == fg.FG_EINVAL, bad
    for bad in (dict(cols=16385), dict(rows=1 << 29), dict(x_ld=1 << 57)):
        assert call(**bad) == fg.FG_EUNSUPPORTED, bad
    assert call(rows=0, x=None, y=None) == fg.FG_OK


def test_layer_norm_bwd_refusals(L):
    d0 = dict(rows=64, cols=40)
    need = fg.layer_norm_workspace_bytes(fg.NormDesc.make(**d0))
    assert need > 0
    assert fg.layer_norm_workspace_bytes(fg.NormDesc.make(4, 20000)) == 0
    assert fg.layer_norm_workspace_bytes(fg.NormDesc.make(4, 0)) == 0

    def call(none=False, dy=at(0), x=at(1), packed=None, stats=at(2), w=at(3), add=at(4),
             dx=at(5), dw=at(6), db=at(7), flag=at(8), ws=at(9), ws_bytes=need, **kw):
        d = fg.NormDesc.make(**{**d0, **kw})
        return L.layer_norm_bwd(None if none else ctypes.byref(d), dy, x, packed, stats, w, add,
                                dx, dw, db, flag, ws, ws_bytes, None)

    assert call(none=True) == fg.FG_EINVAL
    for bad in (dict(dy=None), dict(x=None), dict(stats=None), dict(packed=at(10)),
                dict(dx=None, dw=None, db=None), dict(x=None, packed=at(1) + 4), dict(dx=at(1)),
                dict(dx=at(0) + 2), dict(dx=at(0), dx_ld=48), dict(dx=at(4) + 16), dict(dw=at(3)),
                dict(dw=at(7)), dict(dw=at(5)), dict(flag=at(5)), dict(ws=at(1)), dict(flag=at(2)),
                dict(flag=at(8) + 2), dict(dx=at(5) + 1), dict(stats=at(2) + 4),
                dict(x=None, packed=at(5)), dict(eps=0.0), dict(x_ld=8)):
        assert call(**bad) == fg.FG_EINVAL, bad
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=at(9) + 8)):
        assert call(**bad) == fg.FG_EWORKSPACE, bad
    assert call(cols=16385) == fg.FG_EUNSUPPORTED
    # nothing to do
    assert call(rows=0, dy=None, x=None, stats=None, dw=None, db=None, ws=None) == fg.FG_OK


def test_bindings_check_tensors():
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)
    d = fg.NormDesc.make(24, 8)
    with pytest.raises(ValueError, match="element type"):
        fg.layer_norm_fwd(d, h(24, 8).float(), h(24, 8), stream=0)
    with pytest.raises(ValueError, match="shape"):
        fg.layer_norm_fwd(d, h(24, 9), h(24, 8), stream=0)
    with pytest.raises(ValueError, match="strides"):
        fg.layer_norm_fwd(d, h(24, 16)[:, :8], h(24, 8), stream=0)
    # tensors in host memory never reach the library
    with pytest.raises(ValueError, match="GPU"):
        fg.layer_norm_fwd(d, h(24, 8), h(24, 8), stream=0)
    with pytest.raises(ValueError, match="packed"):
        fg.act8_unpack(fg.Act8Desc.make(24, 8), torch.zeros(10, dtype=torch.uint8), h(24, 8),
                       stream=0)
    with pytest.raises(ValueError, match="GPU"):
        fg.act8_pack(fg.Act8Desc.make(24, 8), h(24, 8), torch.zeros(2000, dtype=torch.uint8),
                     stream=0)
    none = torch.empty(0, 8, dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        fg.layer_norm_fwd(fg.NormDesc.make(0, 8), none, none, stream=0)
