"""layer_norm_fwd and layer_norm_bwd against the formulas in 64 bits: every team of lanes,
type and stride, the input itself or its 8-bit checkpoint, outputs left out, in place, rows
of constants, infinities and NaN, many and few rows, graphs, other streams, offsets past 32
bits.

Bounds, with u = 2^-24 (fp32) and h = half a step of the result's type. A row's sum of C terms is
at most 32 sums in a lane, 6 across lanes and 8 across waves, so it is off by at most 46 u times
the terms' magnitudes; with the factor 1/C (2 u): 48 u.
  mean: 48 u mean|x|.
  x - mean: u|x - mean| and the mean's error m.
  variance v: its terms are off by 2 (u |d| + m) |d| + u d^2, the sum by 48 u: relative
    51 u + 2 m / sqrt(v + eps) (+ (m / sqrt(v + eps))^2). rstd: half that, and 3 u for eps, root
    and quotient (each within u, the quotient of the device's division within 2 u).
  y: 3 u for the products and the sum of each magnitude, and h|y|.
  dx, from the given mean and rstd: xh is within 2 u; g within u; mean(g) within 49 u of a1 =
    mean|g|, mean(g xh) within 52 u of a2; three products and sums (4 u) of |g| + |s1| + |xh s2|;
    the last sum u; h.
  dweight: a column's sum of n rows is at most n sums in a lane (fewer), 6 across teams, 64 + 8
    across workgroups: (n + 78 + 4) u of the terms' magnitudes, and h.
Subnormal results of fp16 and bf16: half their spacing.
"""
import pytest
import torch

import paper_1909_11150_amd as fg
from oracle import block as B

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
EPS = 1e-5
# rows, cols, stride, elements before the first
SHAPES = [(1, 1, 1, 0), (1, 7, 7, 0), (3, 8, 9, 1), (2, 31, 31, 0), (5, 64, 64, 0), (33, 65, 65, 3),
          (17, 100, 104, 0), (64, 256, 1024, 0), (9, 511, 511, 0), (700, 512, 512, 0),
          (6, 513, 520, 1), (40, 1000, 1000, 0), (5, 1025, 1025, 0), (4, 2048, 2048, 0),
          (3, 2049, 2049, 0), (7, 4095, 4100, 0), (1, 4096, 4096, 0), (2, 8192, 8192, 0),
          (3, 8193, 8193, 0), (2, 16384, 16384, 0), (1031, 96, 96, 0), (5000, 40, 40, 0),
          (2500, 1536, 1536, 0)]


def rand(rows, cols, ld, dt, lead=0, seed=0, offset=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1009 + rows * 7 + cols)
    t = torch.randn(rows * ld + lead, generator=g, device="cuda") + offset
    t = t.to(dt)
    return t[lead:].view(rows, ld)[:, :cols], t


def half(t, v):
    """Half a step of type t at values v."""
    f = torch.finfo(t)
    return v.abs() * f.eps / 2 + f.tiny * f.eps / 2


def near(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert torch.isfinite(got).all(), what
    assert float(off.max()) <= 0, (what, float(off.max()), int(off.argmax()))


def check_fwd(x, w, b, y, stats, dt):
    want, mean, rstd = B.layer_norm(x, w, b, EPS)
    xd = x.double()
    m = 48 * U * xd.abs().mean(1) + U * mean.abs()
    near(stats[:, 0], mean, m + 1e-45, "mean")
    rel = 0.5 * (51 * U + 2 * m * rstd + (m * rstd) ** 2) + 4 * U
    near(stats[:, 1], rstd, rel * rstd, "rstd")
    xh = (xd - mean[:, None]) * rstd[:, None]
    wd = 1.0 if w is None else w.double().abs()
    bd = 0.0 if b is None else b.double().abs()
    tol = wd * (xh.abs() * (rel[:, None] + 4 * U) + (m * rstd)[:, None]) * 1.001 + 2 * U * bd
    near(y, want, tol + half(dt, want.abs() + tol), "y")


def check_bwd(o, dx, dw, db, rows, rstd, add, dt):
    near(dx, o["dx"], _dx_tol(o, rstd, add, dt), "dx")
    for got, k, a in ((dw, "dweight", "aw"), (db, "dbias", "ab")):
        tol = (rows + 82) * U * o[a]
        near(got, o[k], tol + half(dt, o[k].abs() + tol), k)


def _dx_tol(o, rstd, add, dt):
    r = rstd.double()[:, None]
    inner = o["g"].abs() + o["s1"].abs() + (o["xh"] * o["s2"]).abs()
    tol = r * (49 * U * o["a1"] + 54 * U * o["xh"].abs() * o["a2"] + 6 * U * inner)
    tol = tol + U * (o["dx"].abs() + (0 if add is None else add.double().abs()))
    return tol + half(dt, o["dx"].abs() + tol)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_matches_the_formulas(dt, shape):
    rows, cols, ld, lead = shape
    t = TYPES[dt]
    x, _ = rand(rows, cols, ld, t, lead, 1, offset=0.5)
    w, b = rand(1, cols, cols, t, 0, 2, 1.0)[1], rand(1, cols, cols, t, 0, 3)[1]
    dy, _ = rand(rows, cols, ld, t, lead, 4)
    add, _ = rand(rows, cols, cols, t, 0, 5)
    y, ywhole = rand(rows, cols, ld, t, lead, 6)
    dx, dxwhole = rand(rows, cols, ld, t, lead, 7)
    before = ywhole.clone(), dxwhole.clone()
    stats = torch.empty(rows, 2, device="cuda")
    d = fg.NormDesc.make(rows, cols, eps=EPS, dtype=fg.dtype_of(x), x_ld=ld, y_ld=ld, dx_ld=ld)
    n = fg.act8_bytes(rows, cols)
    packed = torch.full((n + 64,), 99, dtype=torch.uint8, device="cuda")
    fg.layer_norm_fwd(d, x, y, weight=w, bias=b, stats=stats, packed=packed)
    check_fwd(x, w, b, y, stats, t)
    bytes_, value = B.checkpoint(x)
    assert torch.equal(packed[:n], bytes_) and bool((packed[n:] == 99).all())
    ws = torch.empty(max(16, fg.layer_norm_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    for kept in (None, packed):
        dw, db = torch.empty_like(w), torch.empty_like(b)
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        fg.layer_norm_bwd(d, dy, stats, x=x if kept is None else None, packed=kept, weight=w,
                          add=add, dx=dx, dweight=dw, dbias=db, found_nonfinite=flag, ws=ws)
        o = B.layer_norm_grad(dy, x if kept is None else value, stats[:, 0], stats[:, 1], w, add)
        check_bwd(o, dx, dw, db, rows, stats[:, 1], add, t)
        assert int(flag) == 0
    for whole, was, out in ((ywhole, before[0], y), (dxwhole, before[1], dx)):
        was[lead:].view(rows, ld)[:, :cols] = out
        assert torch.equal(whole, was)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("shape", [(600, 5001, 5003, 1), (515, 8192, 8192, 0),
                                   (700, 12001, 12001, 0), (300, 16384, 16384, 0)], ids=str)
def test_several_wide_rows_to_a_workgroup(dt, shape):
    test_matches_the_formulas(dt, shape)


@pytest.mark.parametrize("cols", [40, 1000, 4096])
def test_parts_left_out(cols):
    """No weight, bias or sums; each output alone; results in place of dy and of add."""
    rows, t = 37, torch.float16
    x, dy, add = (rand(rows, cols, cols, t, 0, k)[0] for k in (1, 2, 3))
    d = fg.NormDesc.make(rows, cols, eps=EPS)
    y, stats = torch.empty_like(x), torch.empty(rows, 2, device="cuda")
    fg.layer_norm_fwd(d, x, y, stats=stats)
    check_fwd(x, None, None, y, stats, t)
    z = x.clone()
    fg.layer_norm_fwd(d, z, z)               # in place, nothing kept
    assert torch.equal(z, y)
    ws = torch.empty(fg.layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    o = B.layer_norm_grad(dy, x, stats[:, 0], stats[:, 1])
    dx = torch.empty_like(x)
    fg.layer_norm_bwd(d, dy, stats, x=x, dx=dx)
    near(dx, o["dx"], _dx_tol(o, stats[:, 1], None, t), "dx")
    dw, db = (torch.empty(cols, dtype=t, device="cuda") for _ in range(2))
    fg.layer_norm_bwd(d, dy, stats, x=x, dweight=dw, ws=ws)
    fg.layer_norm_bwd(d, dy, stats, x=x, dbias=db, ws=ws)
    check_bwd(o, dx, dw, db, rows, stats[:, 1], None, t)
    inplace = dy.clone()
    fg.layer_norm_bwd(d, inplace, stats, x=x, dx=inplace)
    assert torch.equal(inplace, dx)
    fg.layer_norm_bwd(d, dy, stats, x=x, add=add, dx=dx)
    inplace = add.clone()
    fg.layer_norm_bwd(d, dy, stats, x=x, add=inplace, dx=inplace)
    assert torch.equal(inplace, dx)


def test_slices_of_one_buffer():
    """Input and output beside each other in one wide buffer."""
    _, whole = rand(200, 512, 512, torch.float16)
    whole = whole.view(200, 512)
    before = whole.clone()
    d = fg.NormDesc.make(200, 100, eps=EPS, x_ld=512, y_ld=512)
    stats = torch.empty(200, 2, device="cuda")
    fg.layer_norm_fwd(d, whole[:, 3:103], whole[:, 103:203], stats=stats)
    check_fwd(before[:, 3:103], None, None, whole[:, 103:203], stats, torch.float16)
    before[:, 103:203] = whole[:, 103:203]
    assert torch.equal(whole, before)


@pytest.mark.parametrize("cols", [24, 700, 5000])
def test_constant_rows(cols):
    """No variance: y is the bias, whatever the constant."""
    x = torch.tensor([0.0, 1.0, -3.5, 60000.0], device="cuda").half()[:, None].repeat(1, cols)
    b = rand(1, cols, cols, torch.float16)[1]
    y, stats = torch.empty_like(x), torch.empty(4, 2, device="cuda")
    fg.layer_norm_fwd(fg.NormDesc.make(4, cols, eps=EPS), x, y, bias=b, stats=stats)
    # the mean is off by 48 u |x| at most, and rstd is 1 / sqrt(eps) at most
    tol = 48 * U * x.double().abs() / EPS ** 0.5
    near(y, b.double().expand(4, cols), tol + half(torch.float16, b.double().abs() + tol), "y")
    assert torch.equal(y[0], b)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("cols", [96, 3000])
def test_rows_that_are_no_numbers(kept, cols):
    """An infinity or NaN spoils its row and the columns' sums, no other row; the flag rises."""
    rows = 21
    x, dy = rand(rows, cols, cols, torch.float16, 0, 1)[0], rand(rows, cols, cols,
                                                                 torch.float16, 0, 2)[0]
    x[3, 5], x[20, 0] = float("inf"), float("nan")
    d = fg.NormDesc.make(rows, cols, eps=EPS)
    y, stats, dx = torch.empty_like(x), torch.empty(rows, 2, device="cuda"), torch.empty_like(x)
    packed = torch.empty(fg.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    fg.layer_norm_fwd(d, x, y, stats=stats, packed=packed)
    good = [r for r in range(rows) if r not in (3, 20)]
    check_fwd(x[good], None, None, y[good], stats[good], torch.float16)
    assert not torch.isfinite(y[3]).all() and torch.isnan(y[20]).all()
    ws = torch.empty(fg.layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dw, flag = torch.empty(cols, dtype=torch.float16, device="cuda"), \
        torch.zeros(1, dtype=torch.int32, device="cuda")
    fg.layer_norm_bwd(d, dy, stats, x=None if kept else x, packed=packed if kept else None, dx=dx,
                      dweight=dw, found_nonfinite=flag, ws=ws)
    assert torch.isfinite(dx[good]).all()
    assert torch.isnan(dx[3]).any() and torch.isnan(dx[20]).any()
    assert not torch.isfinite(dw).all() and int(flag) == 1


@pytest.mark.parametrize("cols", [8, 600])
def test_no_rows(cols):
    d = fg.NormDesc.make(0, cols)
    e = torch.empty(0, cols, dtype=torch.float16, device="cuda")
    dw, db = (torch.full((cols,), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    fg.layer_norm_fwd(d, e, e)
    fg.layer_norm_bwd(d, e, torch.empty(0, 2, device="cuda"), x=e, dx=e, dweight=dw, dbias=db,
                      ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert not dw.any() and not db.any()


def test_replays_of_a_graph_on_another_stream():
    """Forward and gradients captured; each replay equals the eager result bit for bit."""
    rows, cols, t = 300, 768, torch.bfloat16
    x, dy = torch.empty(rows, cols, dtype=t, device="cuda"), rand(rows, cols, cols, t, 0, 2)[0]
    w, b = rand(1, cols, cols, t, 0, 3)[1], rand(1, cols, cols, t, 0, 4)[1]
    d = fg.NormDesc.make(rows, cols, dtype=fg.BF16)
    def outputs():
        return dict(y=torch.empty_like(x), stats=torch.empty(rows, 2, device="cuda"),
                    packed=torch.empty(fg.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda"),
                    dx=torch.empty_like(x), dw=torch.empty_like(w), db=torch.empty_like(b),
                    ws=torch.empty(fg.layer_norm_workspace_bytes(d), dtype=torch.uint8,
                                   device="cuda"))
    def go(o):
        fg.layer_norm_fwd(d, x, o["y"], weight=w, bias=b, stats=o["stats"], packed=o["packed"])
        fg.layer_norm_bwd(d, dy, o["stats"], packed=o["packed"], weight=w, dx=o["dx"],
                          dweight=o["dw"], dbias=o["db"], ws=o["ws"])
    a, e = outputs(), outputs()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            go(a)
    for k in range(3):
        x.copy_(torch.randn(rows, cols) + k)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        go(e)
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], e[n]) for n in a if n != "ws")


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes of input: the first and the last rows, and the columns' sums of
    gradients that are 0 but there."""
    cols = 1000
    rows = (1 << 31) // cols + 7
    x = torch.empty(rows, cols, dtype=torch.float16, device="cuda").normal_()
    y, stats = torch.empty_like(x), torch.empty(rows, 2, device="cuda")
    packed = torch.empty(fg.act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    d = fg.NormDesc.make(rows, cols, eps=EPS)
    fg.layer_norm_fwd(d, x, y, stats=stats, packed=packed)
    ends = [0, 1, 2, rows - 3, rows - 2, rows - 1]
    check_fwd(x[ends], None, None, y[ends], stats[ends], torch.float16)
    dy = y.zero_()
    dy[ends] = rand(6, cols, cols, torch.float16)[0]
    dw, db = (torch.empty(cols, dtype=torch.float16, device="cuda") for _ in range(2))
    ws = torch.empty(fg.layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    for kept in (None, packed):
        dx = torch.empty_like(x)
        fg.layer_norm_bwd(d, dy, stats, x=x if kept is None else None, packed=kept, dx=dx,
                          dweight=dw, dbias=db, ws=ws)
        xe = x[ends] if kept is None else B.checkpoint(x[ends])[1]
        o = B.layer_norm_grad(dy[ends], xe, stats[ends, 0], stats[ends, 1])
        check_bwd(o, dx[ends], dw, db, 6, stats[ends, 1], None, torch.float16)
        assert not dx[3:rows - 3].any()
