"""Argument checks of the residual block's calls that need no GPU: every call below fails (or
has nothing to do) before any device call."""
import ctypes
import math
import random

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


def test_act8_widths_whose_rounding_up_passes_31_bits(L):
    top = (1 << 31) - 32
    assert fg.act8_bytes(1, top) == top + top // 32
    for cols in (top + 1, (1 << 31) - 1):
        assert fg.act8_bytes(1, cols) == 0
        d = fg.Act8Desc.make(rows=1, cols=cols)
        for fn in (L.act8_pack, L.act8_unpack):
            assert fn(ctypes.byref(d), None, None, None) == fg.FG_EUNSUPPORTED


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


def test_linear_fwd_refusals(L):
    d0 = dict(rows=64, fan_in=40, fan_out=24, act=fg.ACT_GELU)

    def call(none=False, x=at(0), w=at(1), b=at(2), r=at(3), y=at(4), z=at(5), packed=at(6),
             ws=at(7), ws_bytes=1 << 24, **kw):
        d = fg.LinearDesc.make(**{**d0, **kw})
        return L.linear_fwd(None if none else ctypes.byref(d), x, w, b, r, y, z, packed, ws,
                            ws_bytes, None)

    assert call(none=True) == fg.FG_EINVAL
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(rows=-1), dict(fan_in=0),
                dict(fan_out=0), dict(dtype=3), dict(act=3), dict(act=-1), dict(act=fg.ACT_NONE),
                dict(x_ld=39), dict(w_ld=39), dict(y_ld=23), dict(r_ld=23), dict(z_ld=23),
                dict(dx_ld=39), dict(dw_ld=39), dict(x=at(0) + 1), dict(b=at(2) + 1),
                dict(packed=at(6) + 8), dict(y=at(0)), dict(y=at(1)), dict(y=at(2)), dict(y=at(5)),
                dict(z=at(3)), dict(y=at(3) + 2), dict(y=at(3), y_ld=32), dict(packed=at(1))):
        assert call(**bad) == fg.FG_EINVAL, bad
    for bad in (dict(dtype=fg.F32), dict(rows=1 << 28), dict(fan_in=(1 << 17) + 1),
                dict(fan_out=(1 << 17) + 1), dict(x_ld=1 << 20), dict(rows=1 << 27, fan_out=1024)):
        assert call(**bad) == fg.FG_EUNSUPPORTED, bad
        assert fg.linear_workspace_bytes(fg.LinearDesc.make(
            **{**d0, **{k: v for k, v in bad.items()}}), False) == 0
    assert call(rows=0, x=None, y=None) == fg.FG_OK
    split = dict(rows=64, fan_in=8000, fan_out=24)    # a long sum of few tiles, in parts
    need = fg.linear_workspace_bytes(fg.LinearDesc.make(**split), False)
    if need:
        for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=at(7) + 8)):
            assert call(**split, **bad) == fg.FG_EWORKSPACE


def test_a_training_steps_workspace_serves_its_forward_pass():
    """Whatever the sizes: long sums of few tiles are split forward too."""
    rng = random.Random(3)
    for _ in range(300):
        size = lambda hi: int(math.exp(rng.uniform(0, math.log(hi))))
        for act in (fg.ACT_NONE, fg.ACT_GELU):
            d = fg.LinearDesc.make(size(70000), size(20000), size(20000), act=act)
            assert fg.linear_workspace_bytes(d, True) >= fg.linear_workspace_bytes(d, False)


def test_linear_bwd_refusals(L):
    d0 = dict(rows=64, fan_in=40, fan_out=24, act=fg.ACT_GELU)
    need = fg.linear_workspace_bytes(fg.LinearDesc.make(**d0), True)
    assert need > 0

    def call(none=False, dy=at(0), x=at(1), px=None, w=at(2), z=at(3), pz=None, dx=at(4),
             dw=at(5), db=at(6), flag=at(7), ws=at(8), ws_bytes=need, **kw):
        d = fg.LinearDesc.make(**{**d0, **kw})
        return L.linear_bwd(None if none else ctypes.byref(d), dy, x, px, w, z, pz, dx, dw, db,
                            flag, ws, ws_bytes, None)

    assert call(none=True) == fg.FG_EINVAL
    for bad in (dict(dy=None), dict(x=None), dict(w=None), dict(z=None), dict(px=at(9)),
                dict(pz=at(9)), dict(dx=None, dw=None, db=None), dict(act=fg.ACT_NONE),
                dict(x=None, px=at(9) + 4), dict(z=None, pz=at(9) + 4), dict(dx=at(0)),
                dict(dx=at(2)), dict(dw=at(1)), dict(dw=at(4)), dict(db=at(0)), dict(flag=at(6)),
                dict(flag=at(7) + 1), dict(ws=at(0)), dict(dw=at(8)), dict(dx=at(4) + 1),
                dict(rows=-1), dict(dx_ld=8), dict(x=None, px=at(4))):
        assert call(**bad) == fg.FG_EINVAL, bad
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=at(8) + 8)):
        assert call(**bad) == fg.FG_EWORKSPACE, bad
    assert call(dtype=fg.F32) == fg.FG_EUNSUPPORTED
    assert call(dw_ld=1 << 20) == fg.FG_EUNSUPPORTED


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
