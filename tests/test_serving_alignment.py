"""Pointers that are not aligned to their elements are refused on the host (no GPU needed): an access through
one would fault."""
import ctypes

import pytest

from paper_2002_09049_gb300 import _build, binding

P = ctypes.c_void_p
FAKE = 0x10000       # never dereferenced: what passes the checks fails to launch without a GPU

WS = binding.MPQ_CACHE_WORKSPACE
F32, F16 = 0, 1


def calls(lib):
    """name: (function, arguments by name in order, {argument: its elements' bytes})."""
    mx, kv = binding.mpq_mx_layout(4, 64), binding.mpq_cache_layout(4, 16, 2, 64, 8)
    return {
        "quantize_f32": (lib.mpq_mx_quantize, dict(X=FAKE, t=F32, ld=64, lay=mx, packed=FAKE, s=None), dict(X=4)),
        "quantize_f16": (lib.mpq_mx_quantize, dict(X=FAKE, t=F16, ld=64, lay=mx, packed=FAKE, s=None), dict(X=2)),
        "dequantize": (lib.mpq_mx_dequantize, dict(p=FAKE, lay=mx, Y=FAKE, t=F32, ld=64, s=None), dict(Y=4)),
        "linear": (lib.mpq_mx_linear, dict(xl=mx, X=FAKE, wl=mx, W=FAKE, bias=FAKE, Y=FAKE, t=F16, ld=4, s=None),
                   dict(bias=4, Y=2)),
        "write": (lib.mpq_cache_write, dict(K=FAKE, V=FAKE, t=F16, lt=128, lh=64, T=3, slots=FAKE, lay=kv,
                                            codes=FAKE, scales=FAKE, s=None), dict(K=2, V=2, slots=8, scales=4)),
        "read": (lib.mpq_cache_read, dict(slots=FAKE, T=3, lay=kv, codes=FAKE, scales=FAKE, K=FAKE, V=FAKE, t=F16,
                                          s=None), dict(slots=8, scales=4)),
        "attention": (lib.mpq_cache_attention, dict(Q=FAKE, t=F16, st=256, B=2, heads=4, lay=kv, codes=FAKE,
                                                    scales=FAKE, table=FAKE, cols=3, lens=FAKE, scale=0.1, window=0,
                                                    O=FAKE, lse=FAKE, ws=FAKE, n=WS, s=None),
                      dict(Q=2, table=4, lens=4, lse=4)),
    }


@pytest.mark.parametrize("name", ["quantize_f32", "quantize_f16", "dequantize", "linear", "write", "read",
                                  "attention"])
def test_misaligned_pointers_are_refused(name):
    _build.build()
    fn, args, elements = calls(binding.load())[name]
    for arg, size in elements.items():
        for off in {1, size // 2}:
            assert fn(*{**args, arg: FAKE + off}.values()) == 1, (arg, off)
            assert b"aligned" in binding.load().mpq_last_error()
