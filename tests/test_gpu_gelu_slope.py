"""gelu's slope at negative z, relative to its terms: linear_bwd of one row, whose dbias is
dy * slope(z) rounded once, and (with the identity for w) whose dx is dz.

Bounds, with u = 2^-24 and h half a step of the type (relative, or of its subnormals). The slope
is Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi):
  Phi(z), z < 0   6.2e-6 (the polynomial's 5.7e-6, roundings) + 2 u z^2 (the exponent's rounding)
                  of itself
  the other term  2 u z^2 (its exponent's rounding) + 8 u of itself
  dz              u for their sum, 2 u for the product with dy; h. (dx: of a 16-bit dz by 1.)
"""
import math

import pytest
import torch

import paper_1909_11150_amd as fg

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def half(t, v):
    f = torch.finfo(t)
    return v.abs() * f.eps / 2 + f.tiny * f.eps / 2


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1536), (1, 1531), (9, 1536)])
def test_negative_z(dt, rows, cols, kept):
    t = TYPES[dt]
    # -6 .. 0 in steps of 2^-8 (bf16 holds those above 2^-8 of the value only: rounded)
    z = (-6.0 + torch.arange(rows * cols, device="cuda") * (6.0 / 1536)) % -6.0
    z = z.to(t).view(rows, cols).contiguous()
    # large enough that fp16's spacing of small numbers hides nothing; powers of two
    dy = torch.full_like(z, 2.0 ** 15)
    d = fg.LinearDesc.make(rows, cols, cols, dtype=fg.dtype_of(z), act=fg.ACT_GELU)
    packed = None
    if kept:
        packed = torch.empty(fg.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        a = fg.Act8Desc.make(rows, cols, dtype=fg.dtype_of(z))
        fg.act8_pack(a, z, packed)
        fg.act8_unpack(a, packed, z)
    w = torch.eye(cols, device="cuda").to(t)
    dx, db = torch.empty_like(z), torch.empty(cols, dtype=t, device="cuda")
    ws = torch.empty(fg.linear_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    fg.linear_bwd(d, dy, w=w, z=None if kept else z, packed_z=packed, dx=dx, dbias=db, ws=ws)
    v = z.double()
    phi = torch.special.ndtr(v)
    bell = v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    want = dy.double() * (phi + bell)
    tol = phi * (6.2e-6 + 2 * U * v * v) + bell.abs() * (2 * U * v * v + 8 * U)
    tol = dy.double() * tol + 3 * U * want.abs()
    off = (dx.double() - want).abs() / (tol + half(t, want.abs() + tol))
    assert float(off.max()) <= 1, (float(off.max()), float(v.view(-1)[int(off.argmax())]))
    if rows == 1:
        off = (db.double() - want[0]).abs() / (tol + half(t, want.abs() + tol))[0]
        assert float(off.max()) <= 1, (float(off.max()), float(v[0, int(off.argmax())]))
