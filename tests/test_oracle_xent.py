"""The cross-entropy oracle: its values against NumPy's arithmetic row by row, its
gradients against differences, masked and empty rows."""
import numpy as np
import pytest
import torch

from oracle.xent import xent


def _case(t=7, h=5, v=11, seed=0):
    rng = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s))
    return f(t, h), f(v, h), torch.from_numpy(rng.integers(0, v, t)), \
        torch.from_numpy(rng.uniform(-1, 2, t))


def test_rows_one_by_one():
    h, w, t, wt = _case()
    t[2], t[5] = -100, 11
    o = xent(h, w, t, wt, mean=False)
    for i in range(7):
        z = [sum(float(a) * float(b) for a, b in zip(h[i], row)) for row in w]
        want = 0.0 if i in (2, 5) else float(wt[i]) * (np.log(np.sum(np.exp(z))) - z[int(t[i])])
        assert float(o["loss"][i]) == pytest.approx(want, rel=1e-12, abs=1e-12)
    assert float(o["totals"][1]) == pytest.approx(float(wt.sum() - wt[2] - wt[5]))


@pytest.mark.parametrize("mean", [False, True])
def test_gradients_against_differences(mean):
    h, w, t, wt = _case()
    t[1] = -1
    wt[4] = 0.0

    def value(h, w):
        o = xent(h, w, t, wt, mean=mean)
        return 3.0 * float(o["totals"][0] / (o["totals"][1] if mean else 1.0))

    o = xent(h, w, t, wt, scale=3.0, mean=mean)
    e = 1e-6
    for arr, grad in ((h, o["dh"]), (w, o["dw"])):
        for i in range(arr.shape[0]):
            for j in range(arr.shape[1]):
                keep = float(arr[i, j])
                arr[i, j] = keep + e
                up = value(h, w)
                arr[i, j] = keep - e
                down = value(h, w)
                arr[i, j] = keep
                # central differences: error e^2 of the third derivative, and 64-bit
                # roundings of the value over 2e
                assert float(grad[i, j]) == pytest.approx((up - down) / (2 * e), abs=1e-7)


def test_no_live_row():
    h, w, t, _ = _case()
    h[:] = float("nan")
    o = xent(h, w, torch.full_like(t, -100), mean=True)
    for k in ("loss", "lse", "totals", "dh", "dw"):
        assert float(o[k].abs().sum()) == 0.0
