"""The quotients of the cache's codes (no GPU): where the elements and the row's largest have 11 bits or
fewer (fp16, bf16), one correction of x r, r the rounded reciprocal of the scale, is the correctly rounded
x / s.  All pairs within a factor of 2^11 are tried; what is smaller has code 0 either way (x / s < 0.1)."""
import numpy as np
import pytest


@pytest.mark.parametrize("qmax", [127, 7])
def test_one_correction_is_the_quotient(qmax):
    f32 = np.float32
    m = np.arange(1024, 2048, dtype=np.float32) / f32(1024)
    x = np.concatenate([m * f32(2.0 ** -e) for e in range(12)])
    for amax in m:
        s = amax * (f32(1) / f32(qmax))
        r = f32(1) / s
        v = x[x <= amax]
        y = v * r
        # the fused operations in 64 bits: the products are exact there, and so is the remainder
        rest = v.astype(np.float64) - y.astype(np.float64) * np.float64(s)
        y1 = (y.astype(np.float64) + rest * np.float64(r)).astype(np.float32)
        assert np.array_equal(y1, v / s)
