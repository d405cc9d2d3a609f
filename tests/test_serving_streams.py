"""The few-bit attention block on a stream that is not the current one (no GPU: the calls and the streams
are stood for by a record): what a call allocates, it allocates on the stream that uses it."""
import contextlib
import types

import pytest
import torch

from paper_2002_09049_gb300 import serving


class Stream:
    """A stream by name; nothing is enqueued on it."""

    def __init__(self, name, handle):
        self.name, self.cuda_stream = name, handle

    def wait_stream(self, other):
        pass

    def __repr__(self):
        return self.name


@pytest.fixture
def world(monkeypatch):
    """current: the stream that is current; log: (what, stream) in order.  A call's stream argument wins over
    the current one, as in the binding."""
    w = types.SimpleNamespace(current="here", log=[])

    @contextlib.contextmanager
    def stream(s):
        before, w.current = w.current, s
        yield
        w.current = before

    def call(name, result=None):
        def f(*args, stream=None, **kw):
            w.log.append((name, w.current if stream is None else stream))
            return result(kw) if result else None
        return f

    lay = lambda rows, d: types.SimpleNamespace(rows=rows, d=d, bytes=rows * d)
    monkeypatch.setattr(serving, "binding", types.SimpleNamespace(
        MPQ_CACHE_WORKSPACE=64, mpq_mx_layout=lay, mpq_mx_quantize=call("quantize"),
        mpq_mx_linear=call("linear", lambda kw: kw["Y"]), mpq_cache_write=call("write"),
        mpq_cache_attention=call("attention"), mpq_cache_read=call("read")))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    make = serving.FewBitAttention._make_buffers
    monkeypatch.setattr(serving.FewBitAttention, "_make_buffers",
                        lambda self, B: (w.log.append(("buffers", w.current)), make(self, B))[1])
    w.block = b = object.__new__(serving.FewBitAttention)
    b.q_heads, b.heads, b.dim, b.d, b.dtype, b.device = 4, 2, 8, 32, torch.bfloat16, torch.device("cpu")
    b.qkv_layout, b.out_layout = lay(64, 32), lay(32, 32)
    b.w_qkv = b.w_out = b.cache = b.codes = b.scales = b.workspace = None
    b._buffers = {}
    return w


def test_prompt(world):
    s = Stream("side", 7)
    world.block.prompt(torch.zeros(5, 32), torch.arange(5), stream=s)
    assert [what for what, _ in world.log] == ["buffers", "quantize", "linear", "write"]
    assert {where for _, where in world.log} == {s}
    world.log.clear()
    world.block.prompt(torch.zeros(5, 32), torch.arange(5))
    assert {where for _, where in world.log} == {"here"}
