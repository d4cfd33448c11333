"""The residual block's oracle: values element by element in Python's arithmetic, gradients
against differences."""
import math

import numpy as np
import pytest
import torch

from oracle import block as B


def _rand(*s, seed=0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(s))


def test_checkpoint_element_by_element():
    x = _rand(3, 70)
    x[0, :32] = 0
    x[1, 3] = 127.75                     # between the last code and the next power of two
    x[2, 64:] = torch.tensor([1.0, 0.5, 1.5 / 64, 2.5 / 64, -0.5 / 64, 1e-9])
    packed, value = B.checkpoint(x)
    assert packed.numel() == 3 * 96 + 3 * 3
    for r in range(3):
        for c0 in (0, 32, 64):
            g = [float(v) for v in x[r, c0:c0 + 32]]
            top = max(abs(v) for v in g)
            e = math.floor(math.log2(top)) if top else -119
            step = 2.0 ** (e - 6)
            assert int(packed[288 + 3 * r + c0 // 32]) == e + 127
            for k, v in enumerate(g):
                q = max(-127, min(127, round(v / step)))      # halves to even
                assert int(packed[96 * r + c0 + k].view(torch.int8)) == q
                assert float(value[r, c0 + k]) == q * step
    assert value[2, 66:68].tolist() == [2 / 64, 2 / 64] and value[2, 68] == 0


def test_checkpoint_of_what_is_no_number():
    x = torch.tensor([[1.0, math.inf, -math.inf, math.nan, -2.0]])
    packed, value = B.checkpoint(x)
    assert packed[:5].view(torch.int8).tolist() == [32, -128, -128, -128, -64]
    assert value[0, 0] == 1 and value[0, 4] == -2 and torch.isnan(value[0, 1:4]).all()
    assert int(packed[32]) == 128


@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
def test_checkpoint_values_are_exact_in_16_bits(kind):
    x = torch.cat([_rand(4, 96) * s for s in (1e-6, 1e-3, 1.0, 3e4)]).to(kind)
    _, value = B.checkpoint(x)
    # (the largest of fp16 are infinite: NaN)
    assert torch.equal(torch.isnan(value), torch.isinf(x.double()))
    assert torch.allclose(value.to(kind).double(), value, rtol=0, atol=0, equal_nan=True)


def _differences(f, at, grad, n=12, e=1e-6, rel=1e-7):
    rng = np.random.default_rng(1)
    flat = at.view(-1)
    for k in rng.choice(flat.numel(), min(n, flat.numel()), replace=False):
        was = flat[k].item()
        flat[k] = was + e
        hi = f()
        flat[k] = was - e
        lo = f()
        flat[k] = was
        assert float(grad.reshape(-1)[k]) == pytest.approx((hi - lo) / (2 * e), rel=rel, abs=1e-7)


def test_layer_norm_rows_and_gradients():
    x, w, b, dy, add = _rand(5, 9), _rand(9, seed=1), _rand(9, seed=2), _rand(5, 9, seed=3), \
        _rand(5, 9, seed=4)
    y, mean, rstd = B.layer_norm(x, w, b, 1e-3)
    for r in range(5):
        v = x[r].tolist()
        m = sum(v) / 9
        s = 1 / math.sqrt(sum((u - m) ** 2 for u in v) / 9 + 1e-3)
        assert y[r].tolist() == pytest.approx([(u - m) * s * float(w[c]) + float(b[c])
                                               for c, u in enumerate(v)])
    o = B.layer_norm_grad(dy, x, mean, rstd, w, add)
    f = lambda: float((B.layer_norm(x, w, b, 1e-3)[0] * dy).sum() + (x * add).sum())
    _differences(f, x, o["dx"])
    _differences(f, w, o["dweight"])
    _differences(f, b, o["dbias"])


@pytest.mark.parametrize("kind", ["none", "relu", "gelu"])
def test_linear_rows_and_gradients(kind):
    x, w, b, res, dy = _rand(4, 6), _rand(7, 6, seed=1), _rand(7, seed=2), _rand(4, 7, seed=3), \
        _rand(4, 7, seed=4)
    y, z, _ = B.linear(x, w, b, res, kind)
    for r in range(4):
        for c in range(7):
            v = sum(float(p) * float(q) for p, q in zip(x[r], w[c])) + float(b[c])
            a = v if kind == "none" else max(v, 0) if kind == "relu" else \
                0.5 * v * (1 + math.erf(v / math.sqrt(2)))
            assert float(y[r, c]) == pytest.approx(a + float(res[r, c]), abs=1e-12)
    o = B.linear_grad(dy, x, w, z, kind)
    f = lambda: float((B.linear(x, w, b, res, kind)[0] * dy).sum())
    _differences(f, x, o["dx"])
    _differences(f, w, o["dw"])
    _differences(f, b, o["dbias"])


def test_slope_far_out():
    z = torch.tensor([-math.inf, -40.0, 0.0, 40.0, math.inf], dtype=torch.float64)
    assert B.slope(z, "gelu").tolist() == [0, 0, 0.5, 1, 1]
