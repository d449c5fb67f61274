"""The table of rotary frequencies against their formulas with 70 digits (no GPU needed): two units of 2^-64 of a turn.

A frequency is a power, at most two products and a blend in 64-bit significands: with x = ln(1 / w), the power of the rounded exponent is off by x 2^-64 of itself, which is
0.4 2^-64 at most, and each of the other operations by 2^-64 or, the power itself, 2^-63 of a value that is 1 at most; ten of them by 2 pi are 1.6 2^-64 turns, less for all pairs but the first, whose
power is exact.  Cutting the fraction off is one unit more at most."""
from decimal import Decimal as D, getcontext

import pytest

from paper_2607_21042_b200 import binding as B

getcontext().prec = 70
TWO_PI = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_21042_b200 import build
    build.build()


def _power(base, n_rot):
    return [(-D(2 * i) / D(n_rot) * D(base).ln()).exp() for i in range(n_rot // 2)]


def _near(want, units, **kw):
    table, _ = B.op_rope_frequencies(device="cpu", **kw)
    off = [abs(D(t % 2 ** 64) - w / TWO_PI * 2 ** 64) for t, w in zip(table.tolist(), want)]
    assert max(off) <= units, float(max(off))


@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5, 1e7, 10001.3])
def test_powers_and_their_stretches(base):
    for n_rot in range(2, 66, 2):
        w = _power(base, n_rot)
        _near(w, 2, n_rot=n_rot, base=base)
        _near([x / D(40.0) for x in w], 2, n_rot=n_rot, base=base, scaling="linear", factor=40.0)
        if n_rot >= 4:
            _near(_power(D(base) * (D(n_rot) / D(n_rot - 2) * D(8.3).ln()).exp(), n_rot), 2, n_rot=n_rot, base=base, scaling="ntk", factor=8.3)


@pytest.mark.parametrize("base", [10000.0, 500000.0])
@pytest.mark.parametrize("n_rot", [30, 64])
def test_blends(base, n_rot):
    w, factor, original = _power(base, n_rot), D(16.0), D(4096)
    pair = lambda rounds: D(n_rot) * (original / (rounds * TWO_PI)).ln() / (2 * D(base).ln())  # noqa: E731
    first, last = int(pair(D(32)).to_integral_value("ROUND_FLOOR")), int(pair(D(1)).to_integral_value("ROUND_CEILING"))
    assert 0 <= first < last < n_rot
    slow = [min(max(D(i - first) / D(last - first), D(0)), D(1)) for i in range(n_rot // 2)]
    _near([x / factor * s + x * (1 - s) for x, s in zip(w, slow)], 2, n_rot=n_rot, base=base, scaling="yarn", factor=16.0, original=4096)
    fast = [min(max((original * x / TWO_PI - 1) / 3, D(0)), D(1)) for x in w]
    # (the number of turns is 4 at most where it counts, and a third of its rounding comes in)
    _near([x / factor * (1 - s) + x * s for x, s in zip(w, fast)], 2, n_rot=n_rot, base=base, scaling="bands", factor=16.0, original=4096)


@pytest.mark.parametrize("low,high,original", [(1.0, 32.0, 100), (1.0, 1.001, 8192), (3.0, 3.5, 20), (0.01, 50.0, 4096)])
def test_narrow_bands(low, high, original):
    """The number of turns is off by 5 + ln(1 / w), at most 20, last places of itself (a power, three operations); by the band's width it moves the blend, and by r / original the turns."""
    for n_rot in (32, 64):
        w = _power(500000.0, n_rot)
        fast = [min(max((original * x / TWO_PI - D(low)) / (D(high) - D(low)), D(0)), D(1)) for x in w]
        assert any(0 < s < 1 for s in fast) or high - low < 0.01
        _near([x / 8 * (1 - s) + x * s for x, s in zip(w, fast)], 2 + 20 * D(high) ** 2 / (D(original) * (D(high) - D(low))), n_rot=n_rot, base=500000.0, scaling="bands", factor=8.0,
              original=original, low=low, high=high)
