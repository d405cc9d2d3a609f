"""4-bit integer weights, rotation and page tables: what the entry points refuse on the host before they touch
the device, their layouts and the rotation's host side (no GPU needed)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

import _decode_step as ref
from paper_2002_09049_gb300 import _build, binding

P = ctypes.c_void_p
FAKE = 0x10000       # never dereferenced: every call below fails validation on the host first
PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)
F32, F16, BF16 = 0, 1, 2
G4_64 = dict(rows=4, d=64, group=32, zeros=False)


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return binding.load()


@pytest.mark.parametrize("rows,d", [(0, 5), (1, 1), (16, 128), (17, 129), (300, 4096)])
@pytest.mark.parametrize("group", ref.GROUPS)
@pytest.mark.parametrize("zeros", [False, True])
def test_g4_layout(lib, rows, d, group, zeros):
    lay = binding.mpq_g4_layout(rows, d, group, zeros)
    assert ctypes.sizeof(lay) == 7 * 4 + 4 + 8
    assert (lay.rows, lay.d, lay.group, lay.zeros) == (rows, d, group, int(zeros))
    assert lay.row_tiles == -(-rows // 16) and lay.k_tiles == -(-d // 128)
    assert lay.tile_bytes == 1024 + (48 if zeros else 32) * (128 // group) and lay.tile_bytes % 16 == 0
    assert lay.bytes == lay.row_tiles * lay.k_tiles * lay.tile_bytes


@pytest.mark.parametrize("args,status", [
    ((-1, 4, 32, 0), 1), ((4, 0, 32, 0), 1), ((4, (1 << 24) + 1, 32, 0), 3), ((2 ** 31 - 1, 1 << 24, 32, 0), 3),
    ((4, 64, 0, 0), 1), ((4, 64, -32, 0), 1), ((4, 64, 16, 0), 3), ((4, 64, 96, 0), 3), ((4, 64, 256, 0), 3),
    ((4, 64, 32, 2), 1), ((4, 64, 32, -1), 1)])
def test_g4_layout_refuses(lib, args, status):
    lay = binding.G4Matrix()
    assert lib.mpq_g4_layout(*args, ctypes.byref(lay)) == status
    assert lib.mpq_g4_layout(4, 64, 32, 0, None) == 1


def call(fn, defaults):
    return lambda **k: fn(*{**defaults, **k}.values())


def g4_calls(lib):
    lay = binding.mpq_g4_layout(**G4_64)
    return dict(
        quantize=(call(lib.mpq_g4_quantize, dict(X=FAKE, t=F32, ld=64, lay=lay, packed=FAKE, s=None)), dict(X=4)),
        dequantize=(call(lib.mpq_g4_dequantize, dict(packed=FAKE, lay=lay, Y=FAKE, t=F16, ld=64, s=None)),
                    dict(Y=2)),
        linear=(call(lib.mpq_g4_linear, dict(X=FAKE, t=BF16, ldx=64, T=3, lay=lay, W=FAKE, bias=FAKE, Y=FAKE,
                                             yt=F32, ldy=4, s=None)), dict(X=2, bias=4, Y=4)))


def test_g4_calls_refuse(lib):
    calls = g4_calls(lib)
    forged = binding.G4Matrix(4, 64, 32, 0, 1, 1, 1152, 100)        # not one that mpq_g4_layout made
    q, _ = calls["quantize"]
    for bad in (dict(X=None), dict(packed=None), dict(packed=FAKE + 8), dict(ld=63), dict(t=3), dict(t=-1),
                dict(lay=None), dict(lay=forged)):
        assert q(**bad) == 1, bad
    assert q(X=None, packed=None, lay=binding.mpq_g4_layout(0, 64, 32)) == 0
    d, _ = calls["dequantize"]
    for bad in (dict(Y=None), dict(packed=None), dict(packed=FAKE + 8), dict(ld=63), dict(t=7), dict(lay=forged)):
        assert d(**bad) == 1, bad
    f, _ = calls["linear"]
    for bad in (dict(X=None), dict(W=None), dict(Y=None), dict(W=FAKE + 8), dict(ldx=63), dict(ldy=3), dict(t=5),
                dict(yt=5), dict(T=-1), dict(lay=None), dict(lay=forged)):
        assert f(**bad) == 1, bad
    assert f(t=F32) == 3 and f(T=(1 << 20) + 1) == 3
    assert f(T=0, X=None, Y=None) == 0 and f(lay=binding.mpq_g4_layout(0, 64, 32), ldy=0, W=None, Y=None) == 0


@pytest.mark.parametrize("name", ["quantize", "dequantize", "linear"])
def test_g4_misaligned_pointers_are_refused(lib, name):
    fn, elements = g4_calls(lib)[name]
    for arg, size in elements.items():
        for off in {1, size // 2}:
            assert fn(**{arg: FAKE + off}) == 1, (arg, off)
            assert b"aligned" in lib.mpq_last_error()


@pytest.mark.parametrize("freq", [1.0, 1e-4, 10000.0 ** -0.375, -0.7, 6.283185307179586, 1e9, 3e-25, 0.0])
def test_rotation_turns(lib, freq):
    """2^64 freq / 2 pi to the nearest whole number (of exact rationals), whole turns dropped."""
    out = np.empty(1, np.uint64)
    f = np.array([freq], np.float64)
    assert lib.mpq_rotation_turns(f.ctypes.data, 1, out.ctypes.data) == 0
    want = Fraction(freq) / (2 * PI) * 2 ** 64
    off = (int(out[0]) - want) % 2 ** 64
    # half a unit, and a product's rounding below it (2^-53 of 2^64 2^-53 |freq| / 2 pi, twice)
    assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(abs(freq)) / 2 ** 40 + Fraction(1, 2 ** 30)


def test_rotation_turns_refuses(lib):
    out = np.empty(1, np.uint64)
    for f, status in ((np.nan, 2), (np.inf, 2), (-np.inf, 2), (2.0 ** 33, 3), (-2.0 ** 33, 3)):
        a = np.array([f])
        assert lib.mpq_rotation_turns(a.ctypes.data, 1, out.ctypes.data) == status
    assert lib.mpq_rotation_turns(None, 1, out.ctypes.data) == 1
    assert lib.mpq_rotation_turns(out.ctypes.data, -1, out.ctypes.data) == 1
    assert lib.mpq_rotation_turns(None, 0, None) == 0
    assert binding.mpq_rotation([1.0, 0.5], device="cpu").tolist() == [
        round(Fraction(f) / (2 * PI) * 2 ** 64) for f in (1.0, 0.5)]


def rows(**k):
    d = dict(x=FAKE, y=FAKE + 4096, weight=None, heads=4, ld_token=256, ld_head=64, ldy_token=256, ldy_head=64)
    return binding.RotateRows(*{**d, **k}.values())


def test_rotate_refuses(lib):
    f = call(lib.mpq_rotate, dict(q=rows(), k=rows(x=FAKE + 8192, y=FAKE + 16384), type=F16, T=3, dim=64,
                                  positions=FAKE, shift=0, turns=FAKE, rot=64, neighbours=0, norm=0, eps=1e-6,
                                  s=None))
    for bad in (dict(q=None), dict(type=3), dict(T=-1), dict(dim=0), dict(dim=63), dict(rot=63), dict(rot=-2),
                dict(rot=66), dict(neighbours=2), dict(norm=2), dict(norm=1, eps=0.0), dict(norm=1, eps=-1.0),
                dict(positions=None), dict(turns=None), dict(positions=FAKE + 2), dict(turns=FAKE + 4)):
        assert f(**bad) == 1, bad
    assert f(norm=1, eps=float("nan")) == 2 and f(norm=1, eps=float("inf")) == 2
    assert f(T=(1 << 30) + 1) == 3 and f(dim=514, rot=0) == 3 and f(q=rows(heads=65537)) == 3
    for bad in (dict(x=None), dict(y=None), dict(heads=-1), dict(ld_token=-1), dict(ld_head=-1),
                dict(x=FAKE + 1), dict(y=FAKE + 1), dict(weight=FAKE),             # weights without a norm
                dict(ldy_head=63), dict(ldy_token=255),                            # output rows overlap
                dict(y=FAKE, ldy_token=512)):                                      # in place, other strides
        assert f(q=rows(**bad)) == 1, bad
        assert f(k=rows(**bad)) == 1, bad
    assert f(norm=1, q=rows(weight=FAKE + 2)) == 1
    assert f(T=0, q=rows(x=None, y=None), k=None) == 0 and f(q=rows(heads=0, x=None), k=None) == 0


def extend_args():
    at = lambda i: FAKE + i * 4096
    return dict(add=at(0), B=3, page=16, cols=5, lens=at(1), new_lens=at(2), table=at(3), pool=at(4), pages=20,
                count=at(5), new_count=at(6), slots=at(7), positions=at(8), N=10, taken=at(9), s=None)


def trim_args():
    at = lambda i: FAKE + i * 4096
    return dict(keep=at(0), B=3, page=16, cols=5, lens=at(1), new_lens=at(2), table=at(3), pool=at(4), pages=20,
                count=at(5), new_count=at(6), s=None)


def test_pages_refuse(lib):
    for fn, args in ((lib.mpq_pages_extend, extend_args()), (lib.mpq_pages_trim, trim_args())):
        f = call(fn, args)
        pointers = [n for n, v in args.items() if v is not None and v >= FAKE]
        for n in pointers:
            assert f(**{n: None}) == 1, n
            for off in (1, 2):
                assert f(**{n: args[n] + off}) == 1, n
                assert b"aligned" in lib.mpq_last_error()
        for bad in (dict(B=-1), dict(page=0), dict(page=-4), dict(cols=-1), dict(pages=-1)):
            assert f(**bad) == 1, bad
        for bad in (dict(B=binding.MPQ_PAGES_MAX_REQUESTS + 1), dict(page=(1 << 30) + 1, cols=0),
                    dict(page=1 << 20, cols=1025), dict(pages=(1 << 30) + 1)):
            assert f(**bad) == 3, bad
    f = call(lib.mpq_pages_extend, extend_args())
    assert f(N=-1) == 1 and f(N=(1 << 30) + 1) == 3 and f(slots=FAKE + 4) == 1


def test_pages_refuse_overlaps(lib):
    """An output within another array, but for lengths and count updated in place."""
    for fn, args, outs in ((lib.mpq_pages_extend, extend_args(), ("new_lens", "new_count", "table", "slots",
                                                                  "positions", "taken")),
                           (lib.mpq_pages_trim, trim_args(), ("new_lens", "new_count", "pool"))):
        f = call(fn, args)
        sizes = dict(add=12, keep=12, lens=12, new_lens=12, table=60, pool=80, count=8, new_count=8, slots=80,
                     positions=40, taken=12)
        for o in outs:
            for n in sizes:
                if n == o or n not in args or (o, n) in (("new_lens", "lens"), ("new_count", "count")):
                    continue
                assert f(**{o: args[n]}) == 1, (o, n)
                assert b"overlaps" in lib.mpq_last_error()
                assert f(**{o: args[n] + sizes[n] - (sizes[n] % 8 or 8)}) == 1, (o, n)
        assert f(new_lens=args["lens"] + 4) == 1 and f(new_count=args["count"] + 4) == 1
