"""Frequencies in turns against whole-number arithmetic, and refusals of make_rope, on the host."""

import numpy as np
import pytest

PI = 314159265358979323846264338327950288419716939937510582097494459  # times 10^62
BITS = 200


def in_turns(radians):
    """radians / (2 pi) in units of 2^-BITS, rounded down."""
    n, d = float(radians).as_integer_ratio()
    return (n * 10 ** 62 << BITS) // (2 * PI * d)


@pytest.fixture(scope="module")
def lib():
    from paper_2405_06856_gb300 import build
    build.build()
    from paper_2405_06856_gb300 import aladdin as A
    return A


@pytest.mark.parametrize("base", [10000.0, 500000.0, 1e8])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_turns_of_far_positions(lib, base, sign):
    """|p freq| 2^-52 radians (the division's rounding 2^-53, that of 2 pi 2^-54) and, by the last of 64 bits, |p| 2^-64 turns."""
    freq = np.concatenate([base ** (-np.arange(64) / 64), [0.3, 6.0, 7.0, 1e-9, 12345.678]]) * sign
    for f, t in zip(freq, lib.aladdin_rope_turns(freq).tolist()):
        exact, bound = in_turns(f), (in_turns(abs(f)) >> 52) + (1 << BITS - 64)
        for p in (1, -1, 131071, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31):
            off = (p * (t << BITS - 64) - p * exact) % (1 << BITS)
            assert min(off, (1 << BITS) - off) <= abs(p) * (bound + 1), (f, p)


def test_factor_without_scaling(lib):
    """A factor that nothing would use is refused, not left out in silence."""
    from paper_2405_06856_gb300 import worker as W
    for more in (dict(), dict(freq=[1.0, 0.5])):
        with pytest.raises(ValueError, match="factor"):
            W.make_rope(4, factor=8.0, device="cpu", **more)
        rope = W.make_rope(4, factor=1.0, device="cpu", **more)
        assert rope.dim == 4 and rope.scale == 1.0
    assert W.make_rope(4, scaling="linear", factor=8.0, device="cpu").dim == 4
