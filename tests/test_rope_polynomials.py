"""The rotation's sine and cosine, modelled on the host in the kernel's own steps and
constants (read from its source): fp32 products, sums and fused steps, against extended
precision, within the bound that the source states."""
import os
import re

import numpy as np
import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_09681_amd", "csrc",
                      "k_rope.hip")
BOUND = 1.05 * 2.0 ** -23
PI = np.longdouble("3.14159265358979323846264338327950288")


def constants():
    text = open(SOURCE).read()
    body = text[text.index("void sin_cos("):]
    body = body[:body.index("\n}")]
    # (hexadecimal only: the exact halves are written as decimals)
    found = [np.float32(float.fromhex(v)) for v in re.findall(r"-?0x1\.[0-9a-f]+p[-+]?\d+(?=f)", body)]
    assert len(found) == 7, found
    return found


def fma(a, b, c):
    """One rounding to fp32 (the product is exact in 48 bits, the sum in 64 nearly so)."""
    return (np.longdouble(a) * np.longdouble(b) + np.longdouble(c)).astype(np.float32)


def sin_cos(r):
    """Sine and cosine of r / 2^32 turns, |r| <= 2^29."""
    unit, s5, s3, s1, c6, c4, c2 = constants()
    x = r.astype(np.float32) * unit
    y = x * x
    s = fma(y * x, fma(y, fma(y, s5, s3), s1), x)
    c = fma(y * y, fma(y, fma(y, c6, c4), c2), fma(y, np.float32(-0.5), np.float32(1)))
    return s, c


def errors(r):
    s, c = sin_cos(r)
    a = r.astype(np.longdouble) * (2 * PI / 2 ** 32)
    return np.abs(np.longdouble(s) - np.sin(a)), np.abs(np.longdouble(c) - np.cos(a))


@pytest.mark.parametrize("lo", [0, 1 << 20, 1 << 27, 300000000, 492000000, 517000000, 526000000, 528800000, (1 << 29) - (1 << 20)])
@pytest.mark.parametrize("sign", [1, -1])
def test_bound(lo, sign):
    r = sign * np.arange(lo, min(lo + (1 << 20), 1 << 29) + 1, dtype=np.int64)
    for e in errors(r):
        # the angle itself is cut to 32 bits of a turn
        assert float(e.max()) + 2 * np.pi * 2.0 ** -32 * 0.71 <= BOUND, (float(e.max()) * 2 ** 23, int(r[e.argmax()]))


def test_the_bound_is_reached():
    """The largest error over every r (by a sweep of each binade's floats and the ends of their rounding ranges)."""
    sine, cosine = errors(np.array([492334384, 528833456, -526008657], dtype=np.int64))
    assert float(sine.max()) < 0.83 * 2.0 ** -23
    assert 1.02 * 2.0 ** -23 < float(cosine.max()) < BOUND
