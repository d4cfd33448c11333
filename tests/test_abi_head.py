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
