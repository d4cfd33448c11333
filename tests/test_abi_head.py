"""Argument checks of the classification head's calls that need no GPU: every call below
fails (or has nothing to do) before any device call."""
import ctypes

import pytest
import torch

import paper_1909_11150_amd as fg

FAKE = 0x10000  # never dereferenced


@pytest.fixture(scope="module")
def L():
    return fg.lib()


def _drop(**kw):
    base = dict(rows=64, cols=32, p=0.5, seed=1)
    base.update(kw)
    return fg.DropoutDesc.make(**base)


@pytest.mark.parametrize("fn", ["dropout_fwd", "dropout_bwd"])
def test_dropout_refusals(L, fn):
    call = lambda d, x=FAKE, z=None, y=FAKE << 4, c=None: getattr(L, fn)(
        ctypes.byref(d) if d else None, x, z, y, c, None)
    assert call(None) == fg.FG_EINVAL
    assert call(_drop(), x=None) == fg.FG_EINVAL
    assert call(_drop(), y=None) == fg.FG_EINVAL
    for bad in (dict(rows=-1), dict(cols=0), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")),
                dict(dtype=3), dict(dtype=-1), dict(x_ld=31), dict(y_ld=31), dict(z_ld=8),
                dict(x_ld=-32)):
        assert call(_drop(**bad)) == fg.FG_EINVAL, bad
    assert call(_drop(rows=1 << 31, cols=16)) == fg.FG_EUNSUPPORTED     # 2^35 elements
    assert call(_drop(rows=1, cols=1 << 31)) == fg.FG_EUNSUPPORTED
    assert call(_drop(rows=1 << 30, cols=4, x_ld=1 << 40)) == fg.FG_EUNSUPPORTED
    assert call(_drop(), x=FAKE + 1) == fg.FG_EINVAL                    # alignment
    assert call(_drop(dtype=fg.F32), z=FAKE * 2 + 2) == fg.FG_EINVAL
    assert call(_drop(), c=FAKE + 2) == fg.FG_EINVAL
    # overlaps: shifted by an element, another stride, the step count inside y
    assert call(_drop(), x=FAKE, y=FAKE + 2) == fg.FG_EINVAL
    assert call(_drop(x_ld=64), x=FAKE, y=FAKE) == fg.FG_EINVAL
    assert call(_drop(), z=FAKE + 64, y=FAKE) == fg.FG_EINVAL
    assert call(_drop(), x=FAKE << 1, y=FAKE, c=FAKE + 64) == fg.FG_EINVAL
    # slices beside each other that overlap by one column
    assert call(_drop(x_ld=64, y_ld=64), x=FAKE, y=FAKE + 62) == fg.FG_EINVAL
    # nothing to do
    assert call(_drop(rows=0), x=None, y=None) == fg.FG_OK


def test_dropout_binding_checks_tensors():
    x = torch.zeros(4, 6, 8, dtype=torch.float16)
    y = torch.zeros(24, 8, dtype=torch.float16)
    d = lambda **kw: fg.DropoutDesc.make(24, 8, 0.5, 1, **kw)
    with pytest.raises(ValueError, match="element type"):
        fg.dropout_fwd(d(dtype=fg.BF16), x, y, stream=0)
    with pytest.raises(ValueError, match="shape"):
        fg.dropout_fwd(fg.DropoutDesc.make(24, 9, 0.5, 1), x, y, stream=0)
    with pytest.raises(ValueError, match="strides"):
        fg.dropout_fwd(d(x_ld=16), x, y, stream=0)
    with pytest.raises(ValueError, match="strides"):
        fg.dropout_fwd(d(), x.transpose(0, 1), y, stream=0)
    with pytest.raises(ValueError, match="element type"):
        fg.dropout_fwd(d(), x.double(), y, stream=0)
    with pytest.raises(ValueError, match="step_count"):
        fg.dropout_fwd(d(), x, y, step_count=torch.zeros(1), stream=0)
    with pytest.raises(fg.FgError):
        fg.dropout_fwd(fg.DropoutDesc.make(24, 8, 2.0, 1), x, y, stream=0)


def _xent(**kw):
    base = dict(rows=64, hidden=32, vocab=100)
    base.update(kw)
    return fg.XentDesc.make(**base)


# addresses 16 MiB apart
H, W, TG, WT, LOSS, LSE, TOT, DH, DW, FLAG, WS = (0x1000000 * i for i in range(1, 12))


def test_xent_refusals(L):
    big = 1 << 30

    def fwd(d, h=H, w=W, t=TG, wt=None, loss=LOSS, lse=None, tot=None, ws=WS, n=big):
        return L.linear_xent_fwd(ctypes.byref(d) if d else None, h, w, t, wt, loss, lse, tot, ws,
                                 n, None)

    def grad(d, h=H, w=W, t=TG, wt=None, loss=LOSS, lse=None, tot=None, dh=DH, dw=DW, flag=None,
             ws=WS, n=big):
        return L.linear_xent_grad(ctypes.byref(d) if d else None, h, w, t, wt, loss, lse, tot, dh,
                                  dw, flag, ws, n, None)

    for call in (fwd, grad):
        assert call(None) == fg.FG_EINVAL
        for k in ("h", "w", "t", "loss", "ws"):
            assert call(_xent(), **{k: None}) == fg.FG_EINVAL, k
        for bad in (dict(rows=-1), dict(hidden=0), dict(vocab=0), dict(dtype=5), dict(dtype=-1),
                    dict(mean=2), dict(scale=float("inf")), dict(scale=float("nan")),
                    dict(h_ld=31), dict(w_ld=31), dict(dh_ld=31), dict(dw_ld=-1)):
            assert call(_xent(**bad)) == fg.FG_EINVAL, bad
            assert L.fg_linear_xent_workspace_bytes(ctypes.byref(_xent(**bad)), 1) == 0
        for bad in (dict(dtype=fg.F32), dict(rows=1 << 28), dict(hidden=(1 << 16) + 1),
                    dict(vocab=(1 << 22) - 64), dict(h_ld=1 << 20), dict(w_ld=1 << 20)):
            assert call(_xent(**bad)) == fg.FG_EUNSUPPORTED, bad
            assert L.fg_linear_xent_workspace_bytes(ctypes.byref(_xent(**bad)), 0) == 0
        assert call(_xent(), h=H + 1) == fg.FG_EINVAL
        assert call(_xent(), t=TG + 2) == fg.FG_EINVAL
        assert call(_xent(), n=100) == fg.FG_EWORKSPACE
        assert call(_xent(), ws=WS + 8) == fg.FG_EWORKSPACE
        # outputs over inputs, over each other and over the workspace
        assert call(_xent(), loss=H + 8) == fg.FG_EINVAL
        assert call(_xent(), lse=LOSS + 4) == fg.FG_EINVAL
        assert call(_xent(), tot=LOSS + 252) == fg.FG_EINVAL
        assert call(_xent(), h=WS + 256) == fg.FG_EINVAL
    assert grad(_xent(), dh=None, dw=None) == fg.FG_EINVAL
    assert grad(_xent(), dh=H) == fg.FG_EINVAL
    assert grad(_xent(), dw=DH + 64) == fg.FG_EINVAL
    assert grad(_xent(), flag=DW + 4) == fg.FG_EINVAL


def test_xent_workspace(L):
    """Numerators of at most a gibibyte (or 256 rows), whatever the number of rows."""
    need = lambda **kw: L.fg_linear_xent_workspace_bytes(ctypes.byref(_xent(**kw)), 1)
    base = dict(hidden=64, vocab=131072, dtype=fg.BF16)
    few = need(rows=100_000, **base)
    # features' copy 12.8 MB, fp32 sums of dw 33.6 MB, small change
    assert (1 << 30) <= few <= (1 << 30) + (100 << 20)
    assert need(rows=200_000, **base) - few <= 40 << 20
    assert need(rows=16, hidden=64, vocab=4_000_000) <= 3 << 30
    assert L.fg_linear_xent_workspace_bytes(ctypes.byref(_xent()), 0) <= need()
    assert 0 < need(rows=0) <= need()


def test_xent_binding_checks_tensors():
    z = lambda *s, dt=torch.float16: torch.zeros(*s, dtype=dt)
    d = _xent()
    ok = dict(h=z(64, 32), w=z(100, 32), target=z(64, dt=torch.int32), loss=z(64, dt=torch.float32))
    for bad in (dict(h=z(64, 31)), dict(h=z(64, 32, dt=torch.bfloat16)), dict(w=z(99, 32)),
                dict(target=z(64, dt=torch.int64)), dict(loss=z(63, dt=torch.float32)),
                dict(h=z(64, 64)[:, :32])):
        a = dict(ok, **bad)
        with pytest.raises(ValueError):
            fg.linear_xent_fwd(d, a["h"], a["w"], a["target"], a["loss"], stream=0)
    with pytest.raises(fg.FgError):      # no workspace
        fg.linear_xent_fwd(d, ok["h"], ok["w"], ok["target"], ok["loss"], stream=0)
    with pytest.raises(ValueError):
        fg.linear_xent_grad(d, ok["h"], ok["w"], ok["target"], ok["loss"], z(64, 32), z(32, 100),
                            stream=0)
