"""layer_norm_fwd of rows that lie far from zero: constant rows, rows of a large mean and little
variance, rows whose first element is far from the others; against the formulas in 64 bits.

Bounds, with u = 2^-24, h half a step of the result's type, and sums of a row off by at most 48 u
times their terms' magnitudes (as in test_gpu_norm.py):
  first mean: x0 + mean(x - x0), x0 the row's first element: off by e = 50 u mean|x - x0| +
    1.01 u |mean|; by nothing where the row is constant.
  its correction, the mean of d = x - (first mean): off by n = 50 u (mean|x - mean| + e).
  mean: n, and its own rounding, 1.01 u |mean|.
  variance v, the mean of d^2 less the correction's square: 56 u (v + e^2) + 2 e n + n^2.
    rstd: half of that relative to v + eps, and 4 u for eps, root and quotient.
  y: xh by rstd's and 4 u; n and u (|x - mean| + e) times rstd; 2 u |bias|; h.
"""
import pytest
import torch

import paper_1909_11150_amd as fg
from oracle import block as B

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
# every team of lanes, and widths whose fp32 sums of one large value round the most
COLS = [1, 7, 40, 100, 250, 511, 777, 1000, 2048, 4095, 5000, 7680, 8068, 8165, 12001, 16384]


def half(t, v):
    f = torch.finfo(t)
    return v.abs() * f.eps / 2 + f.tiny * f.eps / 2


def near(got, want, tol, what):
    off = (got.double() - want).abs() / tol.clamp_min(1e-300)
    assert torch.isfinite(got).all(), what
    assert float(off.max()) <= 1, f"{what}: {float(off.max()):.3f} of the bound"


def check(x, w, b, eps):
    t, (rows, cols) = x.dtype, x.shape
    y, stats = torch.empty_like(x), torch.empty(rows, 2, device="cuda")
    d = fg.NormDesc.make(rows, cols, eps=eps, dtype=fg.dtype_of(x))
    fg.layer_norm_fwd(d, x, y, weight=w, bias=b, stats=stats)
    # (a row's offset changes nothing: without it the formula's own 64-bit sums, off by up to
    # cols * 2^-53 of their terms, stay far below the bounds, which are 0 for constant rows)
    xd = x.double() - x[:, :1].double()
    want, mean, rstd = B.layer_norm(xd, w, b, eps)
    c = xd - mean[:, None]
    mean = mean + x[:, 0].double()
    apart = xd.abs().mean(1)
    e = torch.where(apart > 0, 50 * U * apart + 1.01 * U * mean.abs(), torch.zeros_like(apart))
    n = 50 * U * (c.abs().mean(1) + e)
    near(stats[:, 0], mean, n + 1.01 * U * mean.abs() + 1e-45, "mean")
    # (2^-149: products below fp32's normal numbers)
    var = 56 * U * (c.square().mean(1) + e * e) + 2 * e * n + n * n + 2.0 ** -149
    rel = 0.5 * var * rstd * rstd * 1.01 + 4 * U
    near(stats[:, 1], rstd, rel * rstd, "rstd")
    rel, e, n, r = (v[:, None] for v in (rel, e, n, rstd))
    tol = (c * r).abs() * (rel + 4 * U) + (n + U * (c.abs() + e)) * r
    if w is not None:
        tol = tol * w.double().abs()
    if b is not None:
        tol = tol + 2 * U * b.double().abs()
    near(y, want, tol + half(t, want.abs() + tol), "y")


def rand(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_constant_rows(dt, cols, eps):
    """No variance: y is the bias, whatever the constant."""
    t = TYPES[dt]
    v = [0.0, 1.0, -3.5, 0.1, 1234.5, 6.0e4, -65504.0, 1e-7, 2048.0]
    x = torch.tensor(v, device="cuda").to(t)[:, None].repeat(1, cols)
    b = rand(cols, seed=cols).to(t)
    check(x, None, b, eps)
    y = torch.empty_like(x)
    fg.layer_norm_fwd(fg.NormDesc.make(len(v), cols, eps=eps, dtype=fg.dtype_of(x)), x, y, bias=b)
    assert torch.equal(y, b.expand_as(y))


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dt,mean,spread", [("f32", 1e4, 0.1), ("f32", -1e6, 1.0), ("f32", 3e3, 1e-3),
                                            ("f16", 3e4, 30.0), ("f16", -6e4, 100.0),
                                            ("bf16", 1e3, 8.0), ("bf16", 1e6, 1e4)])
def test_rows_of_a_large_mean(dt, mean, spread, cols):
    t = TYPES[dt]
    x = (mean + spread * rand(9, cols, seed=cols)).to(t)
    w, b = (1 + 0.2 * rand(cols, seed=1)).to(t), (0.2 * rand(cols, seed=2)).to(t)
    check(x, w, b, 1e-5)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows_whose_first_element_lies_far_off(dt, cols):
    t = TYPES[dt]
    x = rand(8, cols, seed=cols)
    x[:, 0] = torch.tensor([1e4, -6e4, 300.0, -5.0, 0.0, 1e-3, 6.5e4, 1.0], device="cuda")
    x[4:] += 100.0
    w, b = (1 + 0.2 * rand(cols, seed=1)).to(t), (0.2 * rand(cols, seed=2)).to(t)
    check(x.to(t), w, b, 1e-5)


def test_rows_that_are_no_numbers_from_their_first_element_on():
    """An infinity or NaN spoils its own row, wherever it stands."""
    for cols in (5, 96, 3000, 9000):
        x = rand(12, cols, seed=cols)
        clean = torch.empty(12, cols, device="cuda")
        d = fg.NormDesc.make(12, cols, dtype=fg.F32)
        fg.layer_norm_fwd(d, x, clean)
        for k, v in enumerate((float("inf"), float("-inf"), float("nan"))):
            x[2 + 3 * k, 0], x[3 + 3 * k, cols - 1] = v, v
        y = torch.empty(12, cols, device="cuda")
        fg.layer_norm_fwd(d, x, y)
        good = [0, 1, 4, 7, 10, 11]
        assert torch.equal(y[good], clean[good])
        assert torch.isnan(y[[2, 3, 5, 6, 8, 9]]).any(1).all()
