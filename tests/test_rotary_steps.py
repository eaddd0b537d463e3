"""Frequencies of rotary positions: the host side, without a GPU."""
import ctypes
import math
from fractions import Fraction

import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import build
from paper_2608_26004_gb300 import serving as S


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build_cuda()


def radians(steps):
    return [2 * math.pi * s / 2.0 ** 64 for s in steps]


# frequencies: a few operations of 2^-53 and the power's own error; and the step's last bit
def close(a, b):
    return abs(a - b) <= 2.0 ** -50 * abs(b) + 2.0 ** -60


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
def test_plain_frequencies(rot, base):
    steps, magnitude = S.rotary_steps(rot, base)
    assert magnitude == 1.0 and len(steps) == rot // 2
    for i, w in enumerate(radians(steps)):
        assert close(w, base ** (-2 * i / rot)), i
    assert steps[0] == int(Fraction(1 / (2 * math.pi)) * 2 ** 64)   # one radian a position


def test_linear_and_base():
    plain = radians(S.rotary_steps(64)[0])
    steps, magnitude = S.rotary_steps(64, scaling=dict(kind="linear", factor=4.0))
    assert magnitude == 1.0 and all(close(w, v / 4) for w, v in zip(radians(steps), plain))
    steps, magnitude = S.rotary_steps(64, scaling=dict(kind="base", factor=4.0))
    got = radians(steps)
    assert magnitude == 1.0 and close(got[0], 1.0) and close(got[-1], plain[-1] / 4)
    assert all(plain[i] / 4 < got[i] < plain[i] for i in range(1, 31))


def test_ramp_and_wavelength():
    rot, base, f, n = 128, 10000.0, 8.0, 4096
    plain = [base ** (-2 * i / rot) for i in range(rot // 2)]
    at = lambda turns: rot * math.log(n / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    assert 0 < lo < hi < rot // 2
    scaling = dict(factor=f, original_length=n, fast=32.0, slow=1.0)
    steps, magnitude = S.rotary_steps(rot, base, dict(scaling, kind="ramp"))
    assert magnitude == pytest.approx(0.1 * math.log(f) + 1.0, rel=2 ** -23)
    for i, w in enumerate(radians(steps)):
        r = 1.0 - min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert close(w, r * plain[i] + (1 - r) * plain[i] / f), i
    steps, magnitude = S.rotary_steps(rot, base, dict(scaling, kind="wavelength", fast=4.0))
    assert magnitude == 1.0
    for i, w in enumerate(radians(steps)):
        r = min(max((n * plain[i] / (2 * math.pi) - 1.0) / 3.0, 0.0), 1.0)
        assert close(w, r * plain[i] + (1 - r) * plain[i] / f), i
    assert S.rotary_steps(rot, base, dict(scaling, kind="ramp", factor=1.0))[1] == 1.0


def test_own_frequencies():
    own = [1.0, 2 * math.pi * 0.25, 7.5, 0.0, -1.0]
    steps, magnitude = S.rotary_steps(10, frequencies=own)
    assert magnitude == 1.0
    for s, w in zip(steps, own):
        turns = Fraction(w / (2 * math.pi))
        exact = turns - math.floor(turns)
        # w / 2 pi to 2^-53 of itself, the fraction exactly, then the step's last bit
        assert abs(Fraction(s, 2 ** 64) - exact) <= Fraction(1, 2 ** 52)
    assert steps[1] == 1 << 62 and steps[3] == 0


def test_refusals():
    for bad in (dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=-2), dict(rotary_dim=8, base=1.0),
                dict(rotary_dim=8, base=math.nan), dict(rotary_dim=8, base=math.inf),
                dict(rotary_dim=8, scaling=dict(kind="linear", factor=0.5)),
                dict(rotary_dim=8, scaling=dict(kind="linear", factor=math.nan)),
                dict(rotary_dim=2, scaling=dict(kind="base", factor=2.0)),
                dict(rotary_dim=8, scaling=dict(kind="base", factor=1e300)),
                dict(rotary_dim=8, scaling=dict(kind="ramp", factor=2.0)),
                dict(rotary_dim=8, scaling=dict(kind="ramp", factor=2.0, original_length=8, fast=1.0, slow=1.0)),
                dict(rotary_dim=8, scaling=dict(kind="wavelength", factor=2.0, original_length=0, fast=4.0, slow=1.0)),
                dict(rotary_dim=4, frequencies=[1.0, math.inf]),
                dict(rotary_dim=4, frequencies=[1.0, 2.0], scaling=dict(kind="linear", factor=2.0))):
        with pytest.raises(A.AsymSpecError):
            S.rotary_steps(**bad)
    for bad in (dict(rotary_dim=4, frequencies=[1.0]), dict(rotary_dim=4, scaling=dict(kind="none")),
                dict(rotary_dim=4, scaling=dict(kind="linear", factor=2.0, fastt=1.0))):
        with pytest.raises(ValueError):
            S.rotary_steps(**bad)
    lib, m, out = S.lib(), ctypes.c_float(), (ctypes.c_uint64 * 4)()
    s = S.RotaryScaling(kind=9, factor=2.0)
    assert lib.asymspec_rotary_steps(8, 1e4, ctypes.byref(s), None, out, ctypes.byref(m)) == A.ERR_INVALID_ARG
    assert lib.asymspec_rotary_steps(8, 1e4, None, None, None, ctypes.byref(m)) == A.ERR_INVALID_ARG
    assert lib.asymspec_rotary_steps(8, 1e4, None, None, out, None) == A.ERR_INVALID_ARG
