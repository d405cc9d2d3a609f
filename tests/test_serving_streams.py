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
    w = types.SimpleNamespace(current="here", log=[], memory=set(), capturing=False)

    @contextlib.contextmanager
    def stream(s):
        before, w.current = w.current, s
        yield
        w.current = before

    def call(name, result=None):
        def f(*args, stream=None, **kw):
            w.given = kw
            w.memory.update(v.data_ptr() for v in (*args, *kw.values()) if torch.is_tensor(v))
            w.log.append((name, w.current if stream is None else stream))
            return result(kw) if result else None
        return f

    lay = lambda rows, d: types.SimpleNamespace(rows=rows, d=d, bytes=rows * d)
    monkeypatch.setattr(serving, "binding", types.SimpleNamespace(
        MPQ_CACHE_WORKSPACE=64, mpq_mx_layout=lay, mpq_mx_quantize=call("quantize"),
        mpq_mx_linear=call("linear", lambda kw: kw["Y"]), mpq_cache_write=call("write"),
        mpq_cache_attention=call("attention"), mpq_cache_read=call("read")))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: w.capturing)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: getattr(w.current, "cuda_stream", 0),
                        raising=False)
    make = serving.FewBitAttention._make_buffers
    monkeypatch.setattr(serving.FewBitAttention, "_make_buffers",
                        lambda self, B: (w.log.append(("buffers", w.current)), make(self, B))[1])
    w.block = b = object.__new__(serving.FewBitAttention)
    b.q_heads, b.heads, b.dim, b.d, b.dtype, b.device = 4, 2, 8, 32, torch.bfloat16, torch.device("cpu")
    b.qkv_layout, b.out_layout = lay(64, 32), lay(32, 32)
    b.w_qkv = b.w_out = b.cache = b.codes = b.scales = b.workspace = None
    b._buffers, b._workspaces = {}, {}
    return w


def test_prompt(world):
    s = Stream("side", 7)
    world.block.prompt(torch.zeros(5, 32), torch.arange(5), stream=s)
    assert [what for what, _ in world.log] == ["buffers", "quantize", "linear", "write"]
    assert {where for _, where in world.log} == {s}
    world.log.clear()
    world.block.prompt(torch.zeros(5, 32), torch.arange(5))
    assert {where for _, where in world.log} == {"here"}


def step(world, B, stream=None):
    """Where a step runs, and the memory that it uses besides its inputs."""
    world.log.clear()
    world.memory.clear()
    x, slots, table, lens = torch.zeros(B, 32), torch.zeros(B), torch.zeros(B, 1), torch.zeros(B)
    world.block.step(x, slots, table, lens, stream=stream)
    assert [what for what, _ in world.log if what != "buffers"] == \
        ["quantize", "linear", "write", "attention", "quantize", "linear"]
    return {where for _, where in world.log}, world.memory - {t.data_ptr() for t in (x, slots, table, lens)}


def test_steps_of_two_streams_share_nothing(world):
    s = Stream("side", 7)
    ran, used = step(world, 3)
    assert ran == {"here"}
    ran, side = step(world, 3, s)
    assert ran == {s} and used and not used & side
    for B in (3, 5):
        step(world, B)
        step(world, B, s)
    assert step(world, 3) == ({"here"}, used) and step(world, 3, s) == ({s}, side)      # nothing made anew
    world.capturing = True
    assert not step(world, 3)[1] & used
