"""The few-bit serving kernels in the checked build (-DMPQ_CHECK_BOUNDS): no index check fails, and every
output equals the normal build's, bit for bit."""
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2002_09049_gb300 import _build, binding

import _checked_serving

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


def test_checked_build(gpu, tmp_path):
    lib = _build.build(checked=True)
    out = tmp_path / "checked.npz"
    r = subprocess.run([sys.executable, os.path.join(HERE, "_checked_serving.py"), str(out)],
                       env=dict(os.environ, MPQ_LIBRARY=lib), capture_output=True, text=True,
                       timeout=900)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    with np.load(out) as z:
        checked = {k: z[k] for k in z.files}
    assert int(checked["build_options"][0]) & binding.MPQ_BUILD_CHECK_BOUNDS
    assert int(checked["flags"][0]) == 0
    normal = _checked_serving.outputs()
    assert int(normal["flags"][0]) == 0
    for key, ref in normal.items():
        assert np.array_equal(checked[key], ref, equal_nan=ref.dtype.kind == "f"), key
