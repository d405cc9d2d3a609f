"""The few-bit serving entry points refuse invalid arguments on the host, before touching the device
(no GPU needed), and lay out their buffers as include/mpq.h says."""
import ctypes

import numpy as np
import pytest

import _serving as ref
from paper_2002_09049_gb300 import _build, binding

P = ctypes.c_void_p
FAKE = P(0x1000)  # never dereferenced: every call below fails validation on the host first
ODD = P(0x1008)


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return binding.load()


@pytest.mark.parametrize("rows,d", [(0, 5), (1, 1), (128, 128), (129, 129), (300, 4096)])
def test_mx_layout(lib, rows, d):
    lay = binding.mpq_mx_layout(rows, d)
    assert ctypes.sizeof(lay) == 5 * 4 + 4 + 2 * 8
    assert lay.d_pad % 128 == 0 and 0 <= lay.d_pad - d < 128
    assert lay.k_tiles * 128 == lay.d_pad and lay.row_tiles == -(-rows // 128)
    assert lay.off_scales % 512 == 0 and lay.off_scales - rows * lay.d_pad // 2 < 512
    assert lay.bytes == lay.off_scales + 512 * lay.row_tiles * lay.k_tiles
    if rows:
        codes = np.zeros((rows, d), np.uint8)
        assert ref.mx_pack(codes, np.zeros((rows, -(-d // 32)), np.uint8)).size == lay.bytes


@pytest.mark.parametrize("rows,d,status", [(-1, 4, 1), (4, 0, 1), (4, (1 << 24) + 1, 3),
                                           (2 ** 31 - 1, 1 << 24, 3)])
def test_mx_layout_refuses(lib, rows, d, status):
    lay = binding.MxMatrix()
    assert lib.mpq_mx_layout(rows, d, ctypes.byref(lay)) == status
    assert lib.mpq_mx_layout(4, 4, None) == 1


def test_mx_calls_refuse(lib):
    lay, other = binding.mpq_mx_layout(4, 64), binding.mpq_mx_layout(8, 96)
    q = lib.mpq_mx_quantize
    assert q(FAKE, 0, 63, lay, FAKE, None) == 1           # rows overlap
    assert q(FAKE, 3, 64, lay, FAKE, None) == 1           # no such type
    assert q(None, 0, 64, lay, FAKE, None) == 1
    assert q(FAKE, 0, 64, lay, None, None) == 1
    assert q(FAKE, 0, 64, lay, ODD, None) == 1            # packed off the 16-byte boundary
    assert q(FAKE, 0, 64, None, FAKE, None) == 1
    assert q(None, 0, 64, binding.mpq_mx_layout(0, 64), None, None) == 0
    forged = binding.MxMatrix(4, 64, 128, 1, 1, 512, 100)  # not one that mpq_mx_layout made
    assert q(FAKE, 0, 64, forged, FAKE, None) == 1
    d = lib.mpq_mx_dequantize
    assert d(FAKE, lay, FAKE, 0, 63, None) == 1
    assert d(FAKE, lay, None, 0, 64, None) == 1
    assert d(FAKE, lay, FAKE, -1, 64, None) == 1
    f = lib.mpq_mx_linear
    assert f(lay, FAKE, other, FAKE, None, FAKE, 0, 8, None) == 1      # d differs
    assert f(lay, FAKE, lay, FAKE, None, FAKE, 0, 3, None) == 1        # ldy < C
    assert f(lay, FAKE, lay, FAKE, None, None, 0, 4, None) == 1
    assert f(lay, ODD, lay, FAKE, None, FAKE, 0, 4, None) == 1
    assert f(lay, FAKE, lay, FAKE, None, FAKE, 7, 4, None) == 1
    assert f(None, FAKE, lay, FAKE, None, FAKE, 0, 4, None) == 1
    empty = binding.mpq_mx_layout(0, 64)
    assert f(empty, None, lay, None, None, None, 0, 4, None) == 0
    assert lib.mpq_last_error() == b""


@pytest.mark.parametrize("args,status", [
    ((-1, 16, 2, 64, 8), 1), ((4, 0, 2, 64, 8), 1), ((4, 24, 2, 64, 8), 3), ((4, 2048, 2, 64, 8), 3),
    ((4, 16, 0, 64, 8), 1), ((4, 16, 1025, 64, 8), 3), ((4, 16, 2, 0, 8), 1), ((4, 16, 2, 80, 8), 3),
    ((4, 16, 2, 64, 1), 1), ((4, 16, 2, 64, 6), 3)])
def test_cache_layout_refuses(lib, args, status):
    lay = binding.KvCache()
    assert lib.mpq_cache_layout(*args, ctypes.byref(lay)) == status


def test_cache_layout(lib):
    lay = binding.mpq_cache_layout(7, 48, 3, 128, 4)
    assert ctypes.sizeof(lay) == 6 * 4 + 2 * 8
    assert lay.row_bytes == 64 and lay.codes_shape == (7, 2, 3, 48, 64)
    assert lay.codes_bytes == 7 * 2 * 3 * 48 * 64 and lay.scales_bytes == 7 * 2 * 3 * 48 * 4


def test_cache_calls_refuse(lib):
    lay = binding.mpq_cache_layout(4, 16, 2, 64, 8)
    w = lambda **k: lib.mpq_cache_write(*{**dict(K=FAKE, V=FAKE, type=0, lt=128, lh=64, T=3, slots=FAKE,
                                                 lay=lay, codes=FAKE, scales=FAKE, s=None),
                                          **k}.values())
    for bad in (dict(K=None), dict(V=None), dict(type=5), dict(lt=-1), dict(lh=-1), dict(T=-1),
                dict(slots=None), dict(lay=None), dict(codes=None), dict(codes=ODD),
                dict(scales=None)):
        assert w(**bad) == 1, bad
    assert w(T=2 ** 30) == 3
    assert w(T=0, K=None, V=None, slots=None) == 0
    r = lambda **k: lib.mpq_cache_read(*{**dict(slots=FAKE, T=3, lay=lay, codes=FAKE, scales=FAKE,
                                                K=FAKE, V=FAKE, type=1, s=None), **k}.values())
    for bad in (dict(slots=None), dict(T=-1), dict(lay=None), dict(codes=None), dict(K=None),
                dict(V=ODD), dict(type=9)):
        assert r(**bad) == 1, bad
    a = lambda **k: lib.mpq_cache_attention(*{**dict(
        Q=FAKE, type=2, stride=256, B=2, heads=4, lay=lay, codes=FAKE, scales=FAKE, table=FAKE, cols=3,
        lens=FAKE, scale=0.1, window=0, O=FAKE, lse=None, ws=FAKE,
        n=binding.MPQ_CACHE_WORKSPACE, s=None), **k}.values())
    for bad in (dict(Q=None), dict(type=4), dict(stride=-1), dict(B=-1), dict(heads=3), dict(heads=0),
                dict(lay=None), dict(codes=None), dict(codes=ODD), dict(table=None), dict(cols=-1),
                dict(lens=None), dict(window=-2), dict(O=None), dict(n=100), dict(ws=ODD)):
        assert a(**bad) == 1, bad
    assert a(type=0) == 3 and a(cols=1 << 27) == 3
    assert a(scale=float("nan")) == 2 and a(scale=float("inf")) == 2
    assert a(B=0, Q=None, lens=None, O=None) == 0
    assert lib.mpq_cache_attention_workspace() == binding.MPQ_CACHE_WORKSPACE
