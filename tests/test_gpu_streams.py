"""The few-bit serving calls on a stream that is not the current one: what a call allocates belongs to the
stream that writes it."""
import gc
import weakref

import pytest
import torch

from paper_2002_09049_gb300 import binding
from paper_2002_09049_gb300.serving import FewBitAttention

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def owner(t):
    """The stream that the allocator keeps t's memory for."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's memory")


def test_outputs_belong_to_the_stream_given(gpu):
    lay = binding.mpq_mx_layout(40, 256)
    kv = binding.mpq_cache_layout(3, 16, 2, 64, 8)
    codes, scales = binding.mpq_cache_empty(kv, DEV)
    x = torch.randn(40, 256, device=DEV)
    k = torch.randn(40, 2, 64, device=DEV)
    slots = torch.arange(40, device=DEV)
    binding.mpq_cache_write(k, k, slots, kv, codes, scales)
    q = torch.randn(1, 4, 64, device=DEV).half()
    table = torch.arange(3, dtype=torch.int32, device=DEV).view(1, 3)
    lens = torch.tensor([40], dtype=torch.int32, device=DEV)
    packed = binding.mpq_mx_quantize(x, lay)
    side = torch.cuda.Stream()

    def calls(stream):
        return [binding.mpq_mx_quantize(x, lay, stream=stream),
                binding.mpq_mx_dequantize(packed, lay, stream=stream),
                binding.mpq_mx_linear(packed, lay, packed, lay, stream=stream),
                *binding.mpq_cache_read(slots, kv, codes, scales, stream=stream),
                binding.mpq_cache_attention(q, table, lens, kv, codes, scales, stream=stream)]

    want = calls(None)
    torch.cuda.synchronize()
    got = calls(side)
    side.synchronize()
    assert [owner(t) for t in got] == [side.cuda_stream] * len(got)
    with torch.cuda.stream(side):
        inside = calls(None) + calls(torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert [owner(t) for t in inside] == [side.cuda_stream] * len(got) + [0] * len(got)
    for a, b in zip(got + inside, want * 3):
        assert torch.equal(a, b)


def block(bits=8):
    gen = torch.Generator(device=DEV).manual_seed(5)
    w = lambda r, c: torch.randn(r, c, generator=gen, device=DEV) / c ** 0.5
    return FewBitAttention(w(12 * 64, 512), w(512, 8 * 64), 8, 2, 64, pages=20, page=16, bits=bits), gen


def test_prompt_on_a_side_stream(gpu):
    """The current stream allocates and writes while the prompt has not yet begun on its own: the cache holds
    what it holds when nothing else runs."""
    blk, gen = block()
    x = torch.randn(300, 512, generator=gen, device=DEV).to(blk.dtype)
    slots = torch.arange(300, device=DEV)
    blk.prompt(x, slots)
    want = blk.tokens(slots)
    blk.codes.zero_()
    blk.scales.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    blk.prompt(x, slots, stream=side)
    spoil = [torch.full((n,), 0x7F, dtype=torch.uint8, device=DEV)
             for n in (300 * 512, 300 * 768 * 2, 300 * 512 * 2) for _ in range(8)]
    torch.cuda.synchronize()
    for a, b in zip(blk.tokens(slots), want):
        assert torch.equal(a, b)
    del spoil


def batch(blk, gen, first, lens):
    """Sequences of lens cached tokens on pages from `first` on: the next step's arguments."""
    table = torch.full((len(lens), 4), -1, dtype=torch.int32, device=DEV)
    slots = []
    for b, n in enumerate(lens):
        need = -(-n // 16)
        table[b, :need] = torch.arange(first, first + need, device=DEV)
        x = torch.randn(n, blk.d, generator=gen, device=DEV).to(blk.dtype)
        blk.prompt(x, torch.arange(n, device=DEV) + first * 16)
        slots.append(first * 16 + n - 1)
        first += need
    x = torch.randn(len(lens), blk.d, generator=gen, device=DEV).to(blk.dtype)
    return (x, torch.tensor(slots, device=DEV), table, torch.tensor(lens, dtype=torch.int32, device=DEV))


def test_overlapping_steps(gpu):
    """Steps of two streams at once, of the same number of tokens: each as alone."""
    blk, gen = block()
    one, two = batch(blk, gen, 0, [40, 3, 60]), batch(blk, gen, 8, [17, 64, 33])
    want = blk.step(*one).clone(), blk.step(*two).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(30):
        y = blk.step(*one).clone()
        z = blk.step(*two, stream=side)
        with torch.cuda.stream(side):
            got.append((y, z.clone()))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[0]) and torch.equal(z, want[1]) for y, z in got)


def replayed(cap, args):
    for name, t in zip(("x", "slots", "table", "lens"), args):
        getattr(cap, name).copy_(t)
    return cap.replay()


def test_captured_step_keeps_its_block(gpu):
    blk, gen = block()
    args = batch(blk, gen, 0, [40, 3, 60])
    want = blk.step(*args).clone()
    cap = blk.capture(3, 4)
    gone = weakref.ref(blk)
    del blk
    gc.collect()
    assert gone() is not None            # (else the replay would read memory that is free)
    torch.cuda.empty_cache()
    spoil = torch.full((1 << 26,), 0x7F, dtype=torch.uint8, device=DEV)
    assert torch.equal(replayed(cap, args), want)
    del spoil


def test_captured_steps_share_nothing(gpu):
    """Two graphs of one size, replayed at once on two streams, and steps between them."""
    blk, gen = block()
    one, two, three = (batch(blk, gen, f, n) for f, n in ((0, [40, 3]), (6, [17, 60]), (14, [33, 20])))
    want = [blk.step(*a).clone() for a in (one, two, three)]
    caps = [blk.capture(2, 4), blk.capture(2, 4)]
    outs = [c.y.data_ptr() for c in caps] + [blk.step(*three).data_ptr()]
    assert len(set(outs)) == 3
    for c, a in zip(caps, (one, two)):
        replayed(c, a)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(30):
        caps[0].replay()
        with torch.cuda.stream(side):
            caps[1].replay()
        y = blk.step(*three)
    torch.cuda.synchronize()
    for got, ref in zip((caps[0].y, caps[1].y, y), want):
        assert torch.equal(got, ref)
