"""mpq_g4_linear_exact refuses on the host what mpq_g4_linear refuses (no GPU needed)."""
import pytest

from paper_2002_09049_gb300 import _build, binding

FAKE = 0x10000       # never dereferenced: every call below fails validation on the host first
F32, BF16 = 0, 2


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return binding.load()


def test_refuses(lib):
    lay = binding.mpq_g4_layout(4, 64, 32)
    forged = binding.G4Matrix(4, 64, 32, 0, 1, 1, 1152, 100)        # not one that mpq_g4_layout made
    defaults = dict(X=FAKE, t=BF16, ldx=64, T=3, lay=lay, W=FAKE, bias=FAKE, Y=FAKE, yt=F32, ldy=4, s=None)
    f = lambda **k: lib.mpq_g4_linear_exact(*{**defaults, **k}.values())
    for bad in (dict(X=None), dict(W=None), dict(Y=None), dict(W=FAKE + 8), dict(ldx=63), dict(ldy=3), dict(t=5),
                dict(yt=5), dict(T=-1), dict(lay=None), dict(lay=forged), dict(X=FAKE + 1), dict(bias=FAKE + 2),
                dict(Y=FAKE + 2)):
        assert f(**bad) == 1, bad
    assert f(t=F32) == 3 and f(T=(1 << 20) + 1) == 3
    assert f(T=0, X=None, Y=None) == 0 and f(lay=binding.mpq_g4_layout(0, 64, 32), ldy=0, W=None, Y=None) == 0


def test_forms_are_refused(lib):
    for bad in ((-1, 16, 1), (4, 16, 1), (2, 0, 1), (2, 8, 1), (2, 24, 1), (2, 272, 1), (2, 256, 0), (2, 256, 3), (2, 256, 16)):
        assert lib.mpq_test_g4_form(*bad) == 1, bad
    assert lib.mpq_test_g4_form(0, 0, 0) == 0
