"""Arguments of rotary positions that pass a float's range, or leave frequencies that do, are refused like others."""
import math

import pytest

from paper_2608_19677_amd import binding as B
from paper_2608_19677_amd import serve

BEYOND = [
    dict(scaling="index", length=math.inf), dict(scaling="turns", length=math.inf), dict(scaling="index", length=4096, high=math.inf),
    dict(scaling="turns", length=4096, high=math.inf), dict(scaling="turns", length=10 ** 400), dict(scaling="index", length=10 ** 400),
    dict(scaling="index", length=4096, high=10 ** 400), dict(scaling="index", length=math.nan), dict(scaling="turns", length=4096, low=math.nan),
    dict(base=10 ** 400), dict(factor=10 ** 400), dict(scaling="linear", factor=5e-324), dict(scaling="base", factor=5e-324),
    dict(scaling="turns", length=1, factor=5e-324), dict(scaling="index", length=4096, factor=5e-324),
]


@pytest.mark.parametrize("kw", BEYOND, ids=[" ".join(f"{a}={b if b != 10 ** 400 else 'huge'}" for a, b in kw.items()) for kw in BEYOND])
def test_frequencies_refuse(kw):
    with pytest.raises(B.CrError):
        serve.rotary_frequencies(64, **kw)
    with pytest.raises(B.CrError):
        serve.Rotary(64, **kw, device="cpu")


def test_frequencies_beyond_a_turns_range_refuse():
    """A base of 10^4 * 10^(-310 * 64 / 62) = 10^-316 has a last frequency of 10^(316 * 62 / 64) = 10^306: a float, but no fraction of a turn
    that can be formed."""
    f = serve.rotary_frequencies(64, scaling="base", factor=1e-310)
    assert 1e305 < f[-1] < 1e307
    for kw in (dict(scaling="base", factor=1e-310), dict(frequencies=f)):
        with pytest.raises(B.CrError, match="fractions of a turn"):
            serve.Rotary(64, **kw, device="cpu")


def test_given_frequencies_and_magnitude_refuse():
    with pytest.raises(B.CrError, match="finite frequencies"):
        serve.Rotary(64, frequencies=[10 ** 400] * 32, device="cpu")
    with pytest.raises(B.CrError, match="magnitude"):
        serve.Rotary(64, magnitude=10 ** 400, device="cpu")


@pytest.mark.parametrize("kw", [dict(scaling="index", length=4096, high=1e308), dict(scaling="index", length=1e10, low=5e-324),
                                dict(scaling="index", length=1e308, low=1e-300, high=1e-299), dict(scaling="turns", length=4096, high=1e308)])
def test_finite_arguments_are_taken(kw):
    """Turns that no pair comes near: all pairs stay, or all are divided, and nothing is refused."""
    plain = serve.rotary_frequencies(64)
    got = serve.rotary_frequencies(64, factor=4.0, **kw)
    assert all(f / 4 <= g * (1 + 1e-12) and g <= f * (1 + 1e-12) for f, g in zip(plain, got))


def test_whole_numbers_are_floats():
    assert serve.rotary_frequencies(64, 10000, "turns", 8, 8192, 1, 4) == serve.rotary_frequencies(64, 10000.0, "turns", 8.0, 8192.0, 1.0, 4.0)
    assert serve.rotary_frequencies(64, 10000, "base", 8) == serve.rotary_frequencies(64, 10000.0, "base", 8.0)
