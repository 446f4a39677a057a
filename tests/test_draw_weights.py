"""The fixed-point weights of a draw, their steps as the kernel makes them, against 64 bits of mantissa -- CPU only."""
import numpy as np
import pytest

LN2, POW, STEP = 0.69314718055994530942, 128, 6755399441055744.0 / 128
long = np.longdouble
TABLE = np.array([float(np.exp2(long(j) / POW)) for j in range(POW)])


def fma(a, b, c):
    return (long(a) * long(b) + long(c)).astype(np.float64)


def weight(d, per, shift):
    """2^shift e^(d / temperature) with per = log2(e) / temperature, before it is rounded to a whole number."""
    y = np.maximum(fma(d, np.full_like(d, per), np.full_like(d, shift)), -2.0)
    z = y + STEP
    nj = (z.view(np.int64) & 0xFFFFFFFF).astype(np.uint32).view(np.int32)
    r = y - (z - STEP)
    p = np.full_like(r, LN2 ** 4 / 24)
    for c in (LN2 ** 3 / 6, LN2 ** 2 / 2, LN2, 1.0):
        p = fma(r, p, np.full_like(r, c))
    return np.ldexp(TABLE[nj & (POW - 1)] * p, nj >> 7)


@pytest.mark.skipif(np.finfo(np.longdouble).nmant < 63, reason="no wider type")
@pytest.mark.parametrize("shift", [51.0, 46.0, 38.0])
@pytest.mark.parametrize("temperature", [1e-3, 0.1, 0.75, 1.0, 3.7, 50.0])
def test_weights_to_the_stated_bound(temperature, shift):
    """y is below 64 in size: its rounding is off by 2^-48 at most, that of 1 / temperature adds 51 * 2^-53, the series
    (r ln 2)^5 / 120 < 2e-15 with r <= 2^-8, and the products some 2^-53 each: times ln 2 and together below 1e-14."""
    t = float(np.float32(temperature))
    rng = np.random.default_rng(int(shift))
    top = np.float32(rng.normal() * 3)
    v = (np.float64(top) - rng.random(50000) * shift * LN2 * t).astype(np.float32)
    d = v[v < top].astype(np.float64) - np.float64(top)
    true = np.exp(long(d) / long(t)) * long(2.0) ** int(shift)
    off = np.abs(long(weight(d, 1.4426950408889634074 / t, shift)) - true)
    assert float((off / true).max()) < 1e-14
