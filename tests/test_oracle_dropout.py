"""The dropout oracle: the generator against the known answers that its paper's authors
publish for ten rounds, the mask's share of kept elements and its independence of the
length, and the definition's gradient against differences."""
import numpy as np
import pytest

from oracle import dropout as D


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))])
def test_known_answers_of_ten_rounds(counter, key, want):
    got = D.philox([np.array([c]) for c in counter], key, 10)
    assert tuple(int(v[0]) for v in got) == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_share_of_kept_elements(p):
    n = 1 << 18
    k = D.keep(n, 1234567, 3, 1, p)
    q = D.threshold(p) / 65536
    # five standard deviations of a binomial share
    assert abs(k.mean() - q) <= 5 * np.sqrt(q * (1 - q) / n)
    assert np.array_equal(D.keep(1001, 1234567, 3, 1, p), k[:1001])


def test_masks_of_other_steps_sites_and_seeds_are_unrelated():
    n = 1 << 16
    base = D.keep(n, 5, 0, 0, 0.5)
    for other in (D.keep(n, 6, 0, 0, 0.5), D.keep(n, 5, 1, 0, 0.5), D.keep(n, 5, 0, 1, 0.5),
                  D.keep(n, 5 + (1 << 32), 0, 0, 0.5)):
        assert abs((base == other).mean() - 0.5) <= 5 * 0.5 / np.sqrt(n)


def test_gradient_against_differences():
    """d/dx of sum(c * (r + keep * x / q)) is c * keep / q."""
    rng = np.random.default_rng(0)
    n, q = 64, D.threshold(0.3) / 65536
    x, c, k = rng.standard_normal(n), rng.standard_normal(n), D.keep(64, 9, 2, 4, 0.3)
    f = lambda v: np.sum(c * np.where(k, v / q, 0.0))
    num = [(f(x + e) - f(x - e)) / 2e-3 for e in 1e-3 * np.eye(n)]
    np.testing.assert_allclose(num, c * k / q, rtol=0, atol=1e-10)
