"""Where operands may lie (no GPU): no kernel loads with a cluster multicast, whose source has to be this
GPU's own memory, which nothing can promise of a pointer that a caller gives; and the serving calls refuse
tensors of more than one device before anything is launched (tensors without memory stand for them)."""
import glob
import os
import re

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2002_09049_gb300 import _build, binding


def _instructions(path):
    """The PTX instructions in a source's string literals, neighbouring literals joined."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for run in re.findall(r'"(?:[^"\\]|\\.)*"(?:\s*"(?:[^"\\]|\\.)*")*', text):
        joined = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', run))
        yield from joined.split(";")


def test_no_multicast_loads():
    paths = [p for e in ("cu", "cuh", "cpp") for p in
             glob.glob(os.path.join(_build.CSRC, "**", f"*.{e}"), recursive=True)]
    copies = [(os.path.basename(p), i) for p in paths for i in _instructions(p) if "cp.async.bulk" in i]
    assert copies                                       # (the scan sees the tile copies)
    assert not [c for c in copies if "multicast" in c[1]]


def _fake(*shape, dtype=torch.float32, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=device)


@pytest.fixture
def tensors(monkeypatch):
    """Every call with its tensors by name, all on cuda:0."""
    from torch._subclasses import fake_tensor
    # (it would make a tensor on the device, which need not exist)
    monkeypatch.setattr(fake_tensor, "init_gpu_context", lambda *a: None, raising=False)
    _build.build()
    lay, kv = binding.mpq_mx_layout(4, 64), binding.mpq_cache_layout(2, 16, 1, 64, 8)
    byte, f32, i32 = torch.uint8, torch.float32, torch.int32
    x, p = ((4, 64), f32), ((lay.bytes,), byte)
    cache = dict(codes=(kv.codes_shape, byte), scales=(kv.scales_shape, f32))
    return {
        "mpq_mx_quantize": (dict(X=x, packed=p), dict(layout=lay)),
        "mpq_mx_dequantize": (dict(packed=p, Y=x), dict(layout=lay)),
        "mpq_mx_linear": (dict(X=p, W=p, bias=((4,), f32), Y=((4, 4), f32)), dict(x_layout=lay, w_layout=lay)),
        "mpq_cache_write": (dict(K=((3, 1, 64), f32), V=((3, 1, 64), f32), slots=((3,), torch.int64), **cache),
                            dict(layout=kv)),
        "mpq_cache_read": (dict(slots=((3,), torch.int64), K=((3, 1, 64), f32), V=((3, 1, 64), f32), **cache),
                           dict(layout=kv)),
        "mpq_cache_attention": (dict(Q=((2, 4, 64), torch.float16), table=((2, 3), i32), lens=((2,), i32),
                                     O=((2, 4, 64), torch.float16), lse=((2, 4), f32),
                                     workspace=((binding.MPQ_CACHE_WORKSPACE,), byte), **cache),
                                dict(layout=kv)),
    }


@pytest.mark.parametrize("name", ["mpq_mx_quantize", "mpq_mx_dequantize", "mpq_mx_linear", "mpq_cache_write",
                                  "mpq_cache_read", "mpq_cache_attention"])
def test_tensors_of_two_devices_are_refused(tensors, name):
    args, rest = tensors[name]
    call = getattr(binding, name)
    for odd in args:
        given = {n: _fake(*shape, dtype=dtype, device="cuda:1" if n == odd else "cuda:0")
                 for n, (shape, dtype) in args.items()}
        with pytest.raises(ValueError, match="device"):
            call(**given, **rest)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["mpq_mx_quantize", "mpq_mx_linear", "mpq_cache_read", "mpq_cache_attention"])
def test_tensors_of_another_than_the_current_device_are_refused(gpu, tensors, name):
    args, rest = tensors[name]
    given = {n: _fake(*shape, dtype=dtype, device="cuda:1") for n, (shape, dtype) in args.items()}
    with pytest.raises(ValueError, match="current device"):
        getattr(binding, name)(**given, **rest)
