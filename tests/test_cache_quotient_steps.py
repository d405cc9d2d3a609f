"""The cache's quotients as the kernel computes them (no GPU): every fused step rounded once to fp32, the
remainder x - y s among them, which the first correction cannot always hold exactly (y = RN(x r) may be 1.5
units in the last place off).  One correction for elements and maxima of 11 bits or fewer (all pairs within a
factor of 2^11; what is smaller has code 0 either way), two for fp32 ones (samples, among them elements next to
the codes' boundaries)."""
import numpy as np
import pytest

f32, f64 = np.float32, np.float64


def fma(a, b, c):
    """fl32(a b + c) of fp32 arrays, rounded once: the product is exact in 64 bits, the sum is rounded to odd
    there (53 bits are enough for that to leave one rounding to 24)."""
    p, c = a.astype(f64) * b.astype(f64), np.asarray(c).astype(f64)
    t = p + c
    v = t - p
    e = (p - (t - v)) + (c - v)                        # what the 64-bit sum lost, exactly
    even = (t.view(np.int64) & 1) == 0
    t = np.where((e != 0) & even, np.nextafter(t, np.where(e > 0, np.inf, -np.inf)), t)
    return t.astype(f32)


def quotient(x, s, r, steps):
    y = x * r
    for _ in range(steps):
        y = fma(fma(-y, s, x), r, y)
    return y


def test_fma_rounds_once():
    """Against exact integers: cases whose 64-bit sum is a tie that its lost part decides."""
    rng = np.random.default_rng(1)
    a = rng.integers(1 << 23, 1 << 24, 20000)
    b = rng.integers(1 << 23, 1 << 24, 20000)
    c = rng.integers(1 << 23, 1 << 24, 20000)
    for shift in (20, 29, 30, 31, 48):                 # a b + c 2^shift, both halves of it near a tie or not
        b[::2] = 1 << 23
        b[1::4] = (1 << 23) + 1
        got = fma(a.astype(f32), b.astype(f32), np.ldexp(c.astype(f32), shift))
        for i in range(0, 20000, 7):
            n = int(a[i]) * int(b[i]) + (int(c[i]) << shift)
            k = n.bit_length() - 24
            q, rest = n >> k, n & ((1 << k) - 1)
            q += rest > 1 << (k - 1) or (rest == 1 << (k - 1) and q & 1)
            assert got[i] == f32(np.ldexp(float(q), k))


@pytest.mark.parametrize("qmax", [127, 7])
def test_one_correction_of_few_bits(qmax):
    m = np.arange(1024, 2048, dtype=f32) / f32(1024)
    x = np.concatenate([m * f32(2.0 ** -e) for e in range(12)])
    inexact = 0
    for amax in m:
        s = amax * (f32(1) / f32(qmax))
        r = f32(1) / s
        v = x[x <= amax]
        y = v * r
        inexact += int((v.astype(f64) - y.astype(f64) * f64(s) != fma(-y, s, v)).sum())
        assert np.array_equal(quotient(v, s, r, 1), v / s)
    assert inexact > 10000                             # (remainders that are rounded do occur)


@pytest.mark.parametrize("qmax", [127, 7])
def test_two_corrections_of_fp32(qmax):
    rng = np.random.default_rng(qmax)
    top = np.exp(rng.uniform(-40, 40, (4000, 1))).astype(f32)
    s = top * (f32(1) / f32(qmax))
    r = f32(1) / s
    half = (s * (rng.integers(0, qmax, (4000, 200)) + 0.5)).astype(f32)
    near = (half.view(np.int32) + rng.integers(-3, 4, half.shape)).astype(np.int32).view(f32)
    for x in (near, (top * rng.random(half.shape)).astype(f32)):
        x = np.minimum(x, top)
        s_, r_ = (np.broadcast_to(t, x.shape) for t in (s, r))
        assert np.array_equal(quotient(x, s_, r_, 2), x / s_)
