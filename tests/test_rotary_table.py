"""The table of frequencies against 60 digits.

avits_rotary_frequencies works in 64-bit floating point and scales by 2^64 at the end.  In turns,
with f = e^-x / 2 pi <= 0.1592: the power is off by one unit (2^-52) of itself, the rounding of its
exponent by x 2^-53, the rounded 2 pi and the division by 2^-53 each, one more division (linear)
2^-53: 0.1592 (2 + 1 + 1 + 1) 2^-53 + 0.1592 max(x e^-x) 2^-53 = (0.80 + 0.06) 2^-53.  A raised base
adds 8 2^-53 of itself times f 2i / width, below 0.05 2^-53 from a base of 10000 on; parts add a
product, a sum and the error of g, which multiplies frequencies of high / original_len turns and
less.  So 2^-53 of a turn per position holds for all of them.
"""
import ctypes
from decimal import Decimal, getcontext

import pytest

import paper_2608_17995_gb300 as av

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def lib():
    av.build()
    return av.lib()


def exact(width, base, scaling, factor, original_len, low, high):
    base, factor = Decimal(base), Decimal(factor)
    if scaling == "base" and width > 2:
        base *= (factor.ln() * width / (width - 2)).exp()
    out = []
    for i in range(width // 2):
        f = (-base.ln() * 2 * i / width).exp() / (2 * PI)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            g = (Decimal(original_len) * f - Decimal(low)) / (Decimal(high) - Decimal(low))
            g = min(Decimal(1), max(Decimal(0), g))
            f = g * f + (1 - g) * f / factor
        out.append(f)
    return out


@pytest.mark.parametrize("width", [2, 10, 64, 96, 128, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1000000.0])
@pytest.mark.parametrize("scaling,factor,length,low,high", [
    ("none", 1.0, 0.0, 1.0, 32.0), ("linear", 8.0, 0.0, 1.0, 32.0), ("linear", 3.0, 0.0, 1.0, 32.0),
    ("base", 4.0, 0.0, 1.0, 32.0), ("parts", 16.0, 8192.0, 1.0, 4.0), ("parts", 4.0, 32768.0, 1.0, 32.0)])
def test_table_within_its_bound(lib, width, base, scaling, factor, length, low, high):
    got = (ctypes.c_uint64 * (width // 2))()
    assert lib.avits_rotary_frequencies(width, base, av._SCALINGS[scaling], factor, length, low, high,
                                        ctypes.addressof(got)) == 0
    want = exact(width, base, scaling, factor, length, low, high)
    worst = max(abs(Decimal(x) / (1 << 64) - w) for x, w in zip(got, want))
    assert worst <= Decimal(2) ** -53
