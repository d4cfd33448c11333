"""linear_fwd and linear_bwd against the formulas in 64 bits: every activation and type, what
is kept of z and x in 16 or 8 bits, sizes from 1 on that nothing divides, strides and
alignments, split sums, every tile, outputs left out, in place, infinities and NaN, graphs,
other streams, offsets past 32 bits.

Bounds, with u = 2^-24, h = half a step of the type (relative, or of its subnormals):
  sums     products of 16-bit values are exact; an fp32 sum of n of them runs in steps of 16,
           parts are joined: 4 (n/16 + 64) u times the sum of the magnitudes
  z        the sum's, and u (|z| + |bias|)
  Phi      relative to Phi(-|z|) 6.2e-6 (the polynomial's 5.7e-6, roundings) + 2 u z^2 (the
           exponent's rounding) up to |z| = 6; beyond, where both are in 0 .. 1e-9, 1e-9; 3 u
  y        1.13 (gelu's largest slope) times z's, |z| times Phi's, 4 u |y|, and h
  dz       |dy| times the slope's error: Phi's, and |z| exp(-z^2/2) / sqrt(2 pi) (2 u z^2 + 8 u);
           2 u |dz|; for the products also h
  dbias    the sum of dz's errors, (rows + 80) u times the magnitudes, and h
  dx, dw   the sums of dz's errors times |w| (|x|), the sum's, and h
  packed_z half a step of its group (a step above 127 of them), by the largest magnitude there
           can be, and z's error
"""
import math

import pytest
import torch

import paper_1909_11150_amd as fg
from oracle import block as B

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
ACTS = {"none": fg.ACT_NONE, "relu": fg.ACT_RELU, "gelu": fg.ACT_GELU}
U = 2.0 ** -24
# rows, in, out
SHAPES = [(1, 1, 1), (1, 7, 3), (2, 8, 8), (3, 5, 40), (5, 40, 5), (17, 33, 65), (33, 100, 64),
          (64, 64, 256), (1, 2048, 520), (24, 1024, 1000), (7, 4095, 333), (130, 257, 129),
          (300, 777, 1003), (513, 512, 768), (1000, 16, 2048), (2000, 1536, 7), (700, 2000, 300),
          (2048, 1024, 1024), (5000, 264, 520), (4097, 1030, 2056)]


def half(t, v):
    f = torch.finfo(t)
    return v.abs() * f.eps / 2 + f.tiny * f.eps / 2


def near(got, want, tol, what):
    assert bool(torch.isfinite(got).all()), what
    off = (got.double() - want).abs()
    worst = float((off / tol.clamp_min(1e-300)).max()) if off.numel() else 0.0
    assert worst <= 1, f"{what}: {worst:.3f} of the bound"


def sum_tol(n):
    return 4 * (n / 16 + 64) * U


class Maker:
    """Matrices in buffers of their own stride and alignment, NaN around them."""

    def __init__(self, dt, seed, wide):
        self.t, self.wide = TYPES[dt], wide
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, rows, cols, scale=1.0):
        extra, lead = (13, 3) if self.wide else (0, 0)
        b = torch.full((rows * (cols + extra) + lead,), math.nan, dtype=self.t, device="cuda")
        v = b[lead:].view(rows, cols + extra)[:, :cols]
        v.copy_(torch.randn(rows, cols, generator=self.g, device="cuda") * scale)
        return v

    def vector(self, n, scale=1.0):
        return (torch.randn(n, generator=self.g, device="cuda") * scale).to(self.t)

    def out(self, rows, cols):
        v = self(rows, cols)
        v.fill_(77.0)
        return v

    def ld(self, cols):
        return cols + 13 if self.wide else 0


def untouched(v):
    """What lies beside the rows is still NaN."""
    if v.stride(0) == v.shape[1] or not v.numel():
        return True
    b = torch.as_strided(v, (v.shape[0] - 1, v.stride(0) - v.shape[1]), (v.stride(0), 1),
                         v.storage_offset() + v.shape[1])
    return bool(torch.isnan(b).all())


def scratch(d, grad):
    return torch.full((max(16, fg.linear_workspace_bytes(d, grad)),), 0xFF, dtype=torch.uint8,
                      device="cuda")   # NaN wherever read


def phi_tol(z):
    """Error of Phi(z), absolute."""
    return torch.special.ndtr(-z.abs()) * (6.2e-6 + 2 * U * z * z) + 3 * U + \
        1e-9 * (z.abs() > 6)


def slope_tol(z, act):
    if act != "gelu":
        return torch.zeros_like(z)
    bell = z.abs() * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return phi_tol(z) + bell * (2 * U * z * z + 8 * U)


def z_tol(z, mag, bias, k):
    return sum_tol(k) * mag + U * (z.abs() + (0 if bias is None else bias.double().abs()))


def check_y(y, x, w, bias, residual, act, t):
    want, z, mag = B.linear(x, w, bias, residual, act)
    tz = z_tol(z, mag, bias, x.shape[1])
    tol = 1.13 * tz + 4 * U * want.abs()
    if act == "gelu":
        tol = tol + z.abs() * phi_tol(z)
    if residual is not None:
        tol = tol + U * residual.double().abs()
    near(y, want, tol + half(t, want.abs() + tol), "y")
    return z, tz


def check_packed(packed, z, tz):
    rows, cols = z.shape
    d = fg.Act8Desc.make(rows, cols, dtype=fg.F32)
    v = torch.empty(rows, cols, device="cuda")
    fg.act8_unpack(d, packed, v)
    wide = -(-cols // 32) * 32
    pad = lambda a: torch.nn.functional.pad(a, (0, wide - cols)).view(rows, -1, 32)
    top = pad(z.abs() + tz).amax(2, keepdim=True)
    e = (torch.frexp(top).exponent - 1).clamp_min(-119)
    step = torch.exp2((e - 6).double())
    tol = pad(tz) + step * torch.where(pad(z.abs() + tz) > 127.4 * step, 1.0, 0.5)
    near(v, z, tol.view(rows, wide)[:, :cols], "packed_z")
    codes = packed[:rows * wide].view(rows, wide)
    assert not codes[:, cols:].any()


def check_grads(dy, x, w, z, act, t, dx=None, dw=None, db=None):
    o = B.linear_grad(dy, x, w, z, act)
    rows, out = dy.shape
    err = dy.double().abs() * slope_tol(z.double(), act) if act != "none" else \
        torch.zeros_like(o["dz"])
    err = err + 2 * U * o["dz"].abs()
    if db is not None:
        tol = err.sum(0) + (rows + 80) * U * o["ab"]
        near(db, o["dbias"], tol + half(t, o["dbias"].abs() + tol), "dbias")
    if act != "none":
        err = err + half(t, o["dz"].abs() + err)
    if dx is not None:
        tol = err @ w.double().abs() + sum_tol(out) * o["ax"]
        near(dx, o["dx"], tol + half(t, o["dx"].abs() + tol), "dx")
    if dw is not None:
        tol = err.t().contiguous() @ x.double().abs() + sum_tol(rows) * o["aw"]
        near(dw, o["dw"], tol + half(t, o["dw"].abs() + tol), "dw")


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_matches_the_formulas(dt, act, shape):
    rows, k, m = shape
    t, wide = TYPES[dt], (rows + k + m) % 2 == 1
    mk = Maker(dt, rows * 31 + k * 7 + m, wide)
    x, w = mk(rows, k), mk(m, k, 1 / math.sqrt(k))
    bias, residual, dy = mk.vector(m, 0.5), mk(rows, m), mk(rows, m)
    y, z = mk.out(rows, m), mk.out(rows, m)
    n = fg.act8_bytes(rows, m)
    packed = torch.full((n + 64,), 99, dtype=torch.uint8, device="cuda")
    d = fg.LinearDesc.make(rows, k, m, dtype=fg.dtype_of(x), act=ACTS[act], x_ld=mk.ld(k),
                           w_ld=mk.ld(k), y_ld=mk.ld(m), r_ld=mk.ld(m), z_ld=mk.ld(m),
                           dx_ld=mk.ld(k), dw_ld=mk.ld(k))
    ws = scratch(d, False)
    kept = act != "none"
    fg.linear_fwd(d, x, w, y, bias=bias, residual=residual, z=z if kept else None,
                  packed_z=packed if kept else None, ws=ws)
    z64, tz = check_y(y, x, w, bias, residual, act, t)
    assert untouched(y)
    if kept:
        near(z, z64, tz + half(t, z64.abs() + tz), "z")
        assert untouched(z) and bool((packed[n:] == 99).all())
        check_packed(packed[:n], z64, tz)
    fg.linear_fwd(d, x, w, y, ws=ws)     # nothing but the product and the activation
    check_y(y, x, w, None, None, act, t)
    # gradients, from z and x themselves and from their checkpoints
    ws = scratch(d, True)
    px = torch.empty(fg.act8_bytes(rows, k), dtype=torch.uint8, device="cuda")
    fg.act8_pack(fg.Act8Desc.make(rows, k, dtype=fg.dtype_of(x), x_ld=mk.ld(k)), x, px)
    for eight in (False, True):
        dx, dw = mk.out(rows, k), mk.out(m, k)
        db, flag = mk.vector(m), torch.zeros(1, dtype=torch.int32, device="cuda")
        zz = None
        if kept and eight:
            pz, zz = B.checkpoint(z)
        elif kept:
            zz = z
        fg.linear_bwd(d, dy, x=None if eight else x, packed_x=px if eight else None, w=w,
                      z=None if eight else zz, packed_z=pz if eight and kept else None, dx=dx,
                      dw=dw, dbias=db, found_nonfinite=flag, ws=ws)
        xx = B.checkpoint(x)[1] if eight else x
        check_grads(dy, xx, w, zz, act, t, dx, dw, db)
        assert untouched(dx) and untouched(dw) and int(flag) == 0


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("shape", [(16641, 72, 1000), (70000, 8, 200), (11140, 41, 1111),
                                   (33000, 512, 384), (98400, 1, 129)], ids=str)
def test_short_sums_of_many_tiles(dt, act, shape):
    """More than a round of the tiles for short sums: 256 outputs by 128 rows, or 128 by 128."""
    test_matches_the_formulas(dt, act, shape)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 48, 64, 65])
@pytest.mark.parametrize("k,m", [(1, 1), (7, 20), (8, 16), (31, 5), (32, 33), (33, 100),
                                 (300, 17), (2048, 1000), (5001, 40)])
def test_few_rows(dt, rows, k, m):
    """Tokens served: sums of every length, and outputs that end inside a workgroup's."""
    t = TYPES[dt]
    mk = Maker(dt, rows * 31 + k * 7 + m, (rows + m) % 2 == 1)
    x, w = mk(rows, k), mk(m, k, 1 / math.sqrt(k))
    bias, residual = mk.vector(m, 0.5), mk(rows, m)
    d = fg.LinearDesc.make(rows, k, m, dtype=fg.dtype_of(x), act=fg.ACT_GELU, x_ld=mk.ld(k),
                           w_ld=mk.ld(k), y_ld=mk.ld(m), r_ld=mk.ld(m), z_ld=mk.ld(m))
    y, z = mk.out(rows, m), mk.out(rows, m)
    fg.linear_fwd(d, x, w, y, bias=bias, residual=residual, z=z, ws=scratch(d, False))
    z64, tz = check_y(y, x, w, bias, residual, "gelu", t)
    near(z, z64, tz + half(t, z64.abs() + tz), "z")
    assert untouched(y) and untouched(z)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows", [1, 32, 33, 64])
@pytest.mark.parametrize("k,m", [(40, 8192), (41, 8193), (1032, 8200)])
def test_few_rows_of_many_outputs(dt, rows, k, m):
    test_few_rows(dt, rows, k, m)


@pytest.mark.parametrize("shape", [(40, 24, 17), (300, 520, 264)], ids=str)
@pytest.mark.parametrize("act", ACTS)
def test_each_output_alone(act, shape):
    """The same bits as together; what a call does not read may be missing."""
    rows, k, m = shape
    mk = Maker("f16", 5, False)
    x, w, dy, z = mk(rows, k), mk(m, k, 1 / math.sqrt(k)), mk(rows, m), mk(rows, m)
    d = fg.LinearDesc.make(rows, k, m, act=ACTS[act])
    z = z if act != "none" else None
    ws = scratch(d, True)
    new = lambda: (mk.out(rows, k), mk.out(m, k), mk.vector(m))
    dx, dw, db = new()
    fg.linear_bwd(d, dy, x=x, w=w, z=z, dx=dx, dw=dw, dbias=db, ws=ws)
    check_grads(dy, x, w, z, act, torch.float16, dx, dw, db)
    ex, ew, eb = new()
    fg.linear_bwd(d, dy, w=w, z=z, dx=ex, ws=ws)
    fg.linear_bwd(d, dy, x=x, z=z, dw=ew, ws=ws)
    fg.linear_bwd(d, dy, z=z, dbias=eb, ws=ws)
    assert torch.equal(dx, ex) and torch.equal(dw, ew) and torch.equal(db, eb)


# sums of each length by every tile of the gradients, in one part and in several
TILES = [(4000, 1000, 17), (2000, 2048, 2056), (5001, 4100, 17), (2000, 2048, 3001),
         (33001, 1030, 129), (8200, 100, 3001), (2000, 3000, 256), (12345, 1030, 384)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("shape", TILES, ids=str)
def test_tiles_of_the_gradients(dt, act, shape):
    test_matches_the_formulas(dt, act, shape)


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("shape", TILES, ids=str)
def test_each_output_alone_by_its_own_tile(act, shape):
    test_each_output_alone(act, shape)


@pytest.mark.parametrize("shape", [(1, 512, 77), (50, 100, 77), (700, 2000, 300),
                                   (3000, 512, 1000)], ids=str)
def test_in_place_of_the_residual(shape):
    rows, k, m = shape
    mk = Maker("bf16", 6, False)
    x, w, r = mk(rows, k), mk(m, k, 1 / math.sqrt(k)), mk(rows, m)
    d = fg.LinearDesc.make(rows, k, m, dtype=fg.BF16, act=fg.ACT_GELU)
    y, ws = mk.out(rows, m), scratch(d, False)
    fg.linear_fwd(d, x, w, y, residual=r, ws=ws)
    fg.linear_fwd(d, x, w, r, residual=r, ws=ws)
    assert torch.equal(y, r)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """The kernels' gradients against differences of the kernels' own loss, in sums over
    directions: sum(dy * (f(v + e d) - f(v - e d))) / 2e = <grad, d>."""
    rows, k, m = 96, 64, 80
    t = torch.float16
    mk = Maker("f16", 8, False)
    x, w, bias, dy = mk(rows, k), mk(m, k, 1 / 8), mk.vector(m), mk(rows, m)
    d = fg.LinearDesc.make(rows, k, m, act=ACTS[act])

    def loss(x, w, b):
        y, z = mk.out(rows, m), mk.out(rows, m)
        fg.linear_fwd(d, x, w, y, bias=b, z=z if act != "none" else None, ws=scratch(d, False))
        return y.double(), z
    y0, z = loss(x, w, bias)
    dx, dw, db = mk.out(rows, k), mk.out(m, k), mk.vector(m)
    fg.linear_bwd(d, dy, x=x, w=w, z=z if act != "none" else None, dx=dx, dw=dw, dbias=db,
                  ws=scratch(d, True))
    for i, (v, grad) in enumerate(((x, dx), (w, dw), (bias, db))):
        # steps that fp16 holds exactly, along the gradient's signs
        e = 2.0 ** -4 * torch.sign(grad.double())
        args = [x, w, bias]
        hi, lo = list(args), list(args)
        hi[i], lo[i] = (v.double() + e * 0.25).to(t), (v.double() - e * 0.25).to(t)
        moved = hi[i].double() - lo[i].double()
        diff = float((dy.double() * (loss(*hi)[0] - loss(*lo)[0])).sum())
        want = float((grad.double() * moved).sum())
        # what the step's length costs: the same difference and gradient in 64 bits
        zh, zl = (B.linear(a[0], a[1], a[2])[1] for a in (hi, lo))
        z64 = B.linear(x, w, bias)[1]
        dz = dy.double() * B.slope(z64, act)
        exact = (dz @ w.double(), dz.t() @ x.double(), dz.sum(0))[i]
        curved = abs(float((dy.double() * (B.act(zh, act) - B.act(zl, act))).sum())
                     - float((exact * moved).sum()))
        # y's rounding in both, independent from element to element: 2^-11 of its size, a random
        # walk, six standard deviations. dz: z kept in fp16 moves gelu's slope by 0.8 (its
        # largest curvature) * 2^-11 |z|, |z| < 4 where there is curvature, so with dz's own
        # rounding 2^-9 of |dy| times what z moved; relu's only where z is 0 in fp16. The
        # gradient's own rounding 2^-11.
        noise = 6 * 2.0 ** -11 * float((dy.double() * y0).norm())
        noise += 2.0 ** -9 * float((dy.double() * (zh - zl)).abs().sum())
        noise += 2.0 ** -11 * float((exact * moved).abs().sum())
        print(f"{i}: off {abs(diff - want):.3g}, curved {curved:.3g}, noise {noise:.3g}, "
              f"of {want:.4g}")
        assert abs(diff - want) <= curved + noise, (i, diff, want)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [5, 200])
def test_rows_that_are_no_numbers(act, rows):
    """They spoil their own row of y, z and dx, and the sums over the rows; the flag rises."""
    k, m = 100, 77
    mk = Maker("f16", 9, False)
    x, w, dy = mk(rows, k), mk(m, k, 0.1), mk(rows, m)
    x[2, 3], x[4, 0] = float("nan"), float("inf")
    d = fg.LinearDesc.make(rows, k, m, act=ACTS[act])
    y, z = mk.out(rows, m), mk.out(rows, m)
    packed = torch.empty(fg.act8_bytes(rows, m), dtype=torch.uint8, device="cuda")
    kept = act != "none"
    fg.linear_fwd(d, x, w, y, z=z if kept else None, packed_z=packed if kept else None,
                  ws=scratch(d, False))
    good = [r for r in range(rows) if r not in (2, 4)]
    check_y(y[good], x[good], w, None, None, act, torch.float16)
    assert torch.isnan(y[2]).all()
    if act == "none":
        assert torch.isinf(y[4]).all()
    for eight in (False, True):
        dx, dw, db = mk.out(rows, k), mk.out(m, k), mk.vector(m)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        fg.linear_bwd(d, dy, x=x, w=w, z=z if kept and not eight else None,
                      packed_z=packed if kept and eight else None, dx=dx, dw=dw, dbias=db,
                      found_nonfinite=flag, ws=scratch(d, True))
        assert torch.isfinite(dx[good]).all()
        assert torch.isnan(dw[:, 3]).all() and int(flag) == 1
        if kept:
            assert torch.isnan(dx[2]).all() and torch.isnan(db).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows", [3, 200])
def test_subnormal_operands(dt, rows):
    """Operands below the type's normal numbers count in full."""
    k, m, t = 72, 40, TYPES[dt]
    mk = Maker(dt, 12, False)
    x, dy = mk(rows, k, torch.finfo(t).tiny / 8), mk(rows, m, torch.finfo(t).tiny / 8)
    w = mk(m, k, 8.0)
    assert bool(((x != 0) & (x.abs() < torch.finfo(t).tiny)).any())
    d = fg.LinearDesc.make(rows, k, m, dtype=fg.dtype_of(x))
    y, dx, dw = mk.out(rows, m), mk.out(rows, k), mk.out(m, k)
    fg.linear_fwd(d, x, w, y, ws=scratch(d, False))
    want, _, mag = B.linear(x, w)
    # (fp32's own subnormals: products and sums below 2^-126 may lose bits of 2^-149)
    tol = sum_tol(k) * mag + k * 2.0 ** -126 * (dt == "bf16")
    near(y, want, tol + half(t, want.abs() + tol), "y")
    fg.linear_bwd(d, dy, x=mk(rows, k), w=w, dx=dx, dw=dw, ws=scratch(d, True))
    o = B.linear_grad(dy, None, w)
    tol = sum_tol(m) * o["ax"] + m * 2.0 ** -126 * (dt == "bf16")
    near(dx, o["dx"], tol + half(t, o["dx"].abs() + tol), "dx")


@pytest.mark.parametrize("m", [8, 300])
def test_far_pre_activations(m):
    """gelu of large and infinite z: 0, z, and no NaN but of NaN."""
    v = [-65504.0, -60.0, -12.0, -5.0, 0.0, 5.0, 60.0, 65504.0]
    x = torch.tensor(v, device="cuda").half()[:, None].repeat(1, 8)
    x[:, 1:] = 0
    w = torch.zeros(m, 8, dtype=torch.float16, device="cuda")
    w[:, 0] = 1
    d = fg.LinearDesc.make(8, 8, m, act=fg.ACT_GELU)
    y, z = torch.empty(8, m, dtype=torch.float16, device="cuda"), \
        torch.empty(8, m, dtype=torch.float16, device="cuda")
    fg.linear_fwd(d, x, w, y, z=z, ws=scratch(d, False))
    assert torch.equal(z, x[:, :1].expand(8, m))
    check_y(y, x, w, None, None, "gelu", torch.float16)
    z[0], z[7] = float("-inf"), float("inf")
    dy, dx, db = torch.ones_like(y), torch.empty_like(x), torch.empty_like(y[0])
    fg.linear_bwd(d, dy, w=w, z=z, dx=dx, dbias=db, ws=scratch(d, True))
    s = dx[:, 0].double() / m
    assert torch.isfinite(dx).all() and torch.isfinite(db).all()
    assert s[0] == 0 and s[1] == 0 and s[6] == 1 and s[7] == 1


def test_no_rows():
    for k, m in ((5, 9), (512, 256)):
        e = lambda n: torch.empty(0, n, dtype=torch.float16, device="cuda")
        for act in (fg.ACT_NONE, fg.ACT_GELU):
            d = fg.LinearDesc.make(0, k, m, act=act)
            w = torch.ones(m, k, dtype=torch.float16, device="cuda")
            fg.linear_fwd(d, e(k), w, e(m))
            dw, db = torch.full_like(w, 3.0), torch.full((m,), 3.0, dtype=w.dtype, device="cuda")
            fg.linear_bwd(d, e(m), x=e(k), w=w, z=e(m) if act else None, dx=e(k), dw=dw, dbias=db,
                          ws=scratch(d, True))
            assert not dw.any() and not db.any()


@pytest.mark.parametrize("shape", [(4, 512, 1000), (600, 1000, 520)], ids=str)
def test_replays_of_a_graph_on_another_stream(shape):
    """Forward and gradients captured; each replay equals the eager result bit for bit."""
    rows, k, m = shape
    mk = Maker("bf16", 3, False)
    x, w, bias, dy = mk(rows, k), mk(m, k, 1 / math.sqrt(k)), mk.vector(m), mk(rows, m)
    d = fg.LinearDesc.make(rows, k, m, dtype=fg.BF16, act=fg.ACT_GELU)

    def outputs():
        return dict(y=mk.out(rows, m), dx=mk.out(rows, k), dw=mk.out(m, k), db=mk.vector(m),
                    pz=torch.empty(fg.act8_bytes(rows, m), dtype=torch.uint8, device="cuda"),
                    px=torch.empty(fg.act8_bytes(rows, k), dtype=torch.uint8, device="cuda"),
                    ws=scratch(d, True), ws1=scratch(d, False))

    def go(o):
        fg.linear_fwd(d, x, w, o["y"], bias=bias, packed_z=o["pz"], ws=o["ws1"])
        fg.act8_pack(fg.Act8Desc.make(rows, k, dtype=fg.BF16), x, o["px"])
        fg.linear_bwd(d, dy, packed_x=o["px"], w=w, packed_z=o["pz"], dx=o["dx"], dw=o["dw"],
                      dbias=o["db"], ws=o["ws"])
    a, e = outputs(), outputs()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            go(a)
    for i in range(3):
        x.copy_(torch.randn(rows, k) * (i + 1))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        go(e)
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], e[n]) for n in a if not n.startswith("ws"))


@pytest.mark.parametrize("k,m", [(1000, 24), (24, 1000)])
def test_offsets_beyond_32_bits(k, m):
    """More than 2^32 bytes of x, or of y: the first and the last rows, and the sums over rows
    of gradients that are 0 but there."""
    rows = (1 << 31) // 1000 + 77
    t = torch.float16
    mk = Maker("f16", 4, False)
    x = torch.empty(rows, k, dtype=t, device="cuda").normal_()
    w = mk(m, k, 1 / math.sqrt(k))
    d = fg.LinearDesc.make(rows, k, m, act=fg.ACT_RELU)
    y = torch.empty(rows, m, dtype=t, device="cuda")
    packed = torch.empty(fg.act8_bytes(rows, m), dtype=torch.uint8, device="cuda")
    fg.linear_fwd(d, x, w, y, packed_z=packed, ws=scratch(d, False))
    ends = [0, 1, 2, rows // 2, rows - 2, rows - 1]
    check_y(y[ends], x[ends], w, None, None, "relu", t)
    z = torch.empty(rows, m, dtype=t, device="cuda")
    fg.act8_unpack(fg.Act8Desc.make(rows, m), packed, z)
    dy = y.zero_()
    dy[ends] = mk(6, m)
    dx, dw, db = torch.empty_like(x), mk.out(m, k), mk.vector(m)
    fg.linear_bwd(d, dy, x=x, w=w, packed_z=packed, dx=dx, dw=dw, dbias=db, ws=scratch(d, True))
    check_grads(dy[ends], x[ends], w, z[ends], "relu", t, dx[ends], dw, db)
    assert not dx[3:rows // 2].any() and not dx[rows // 2 + 1:rows - 2].any()
