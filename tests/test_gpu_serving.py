"""The few-bit attention block (paper_2002_09049_gb300.serving): a step is the six calls it is made of, on
any stream and from a captured graph, and its result is that of the same block in plain fp64 on the
values that the few-bit forms stand for, up to the inputs' 4-bit grids."""
import math

import pytest
import torch

from paper_2002_09049_gb300 import binding
from paper_2002_09049_gb300.serving import FewBitAttention

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def block(bits=8, q_heads=8, heads=2, dim=64, d=512, seed=3):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    w = lambda r, c: torch.randn(r, c, generator=gen, device=DEV) / math.sqrt(c)
    wq, wo = w((q_heads + 2 * heads) * dim, d), w(d, q_heads * dim)
    return FewBitAttention(wq, wo, q_heads, heads, dim, pages=12, page=16, bits=bits), gen


def filled(blk, gen, lens):
    """Prompts of lens[b] - 1 tokens in the cache; (table, lens, next slots)."""
    table = torch.full((len(lens), 3), -1, dtype=torch.int32, device=DEV)
    page = 0
    for b, n in enumerate(lens):
        need = -(-n // 16)
        table[b, :need] = torch.arange(page, page + need, device=DEV)
        if n > 1:
            x = torch.randn(n - 1, blk.d, generator=gen, device=DEV).to(blk.dtype)
            blk.prompt(x, torch.arange(n - 1, device=DEV) + page * 16)
        page += need
    slots = torch.tensor([int(table[b, (n - 1) // 16]) * 16 + (n - 1) % 16
                          for b, n in enumerate(lens)], device=DEV)
    return table, torch.tensor(lens, dtype=torch.int32, device=DEV), slots


@pytest.mark.parametrize("bits", [8, 4])
def test_step_is_its_calls_and_its_graph(gpu, bits):
    blk, gen = block(bits)
    table, lens, slots = filled(blk, gen, [40, 1, 17])
    x = torch.randn(3, blk.d, generator=gen, device=DEV).to(blk.dtype)
    y = blk.step(x, slots, table, lens).clone()
    # the calls, one after another, each with outputs of its own
    xl = binding.mpq_mx_layout(3, blk.d)
    qkv = binding.mpq_mx_linear(binding.mpq_mx_quantize(x, xl), xl, blk.w_qkv, blk.qkv_layout,
                                dtype=blk.dtype)
    torch.cuda.synchronize()
    rows = qkv.view(3, -1, blk.dim)
    K, V = blk.tokens(slots)
    for got, part in ((K, rows[:, 8:10]), (V, rows[:, 10:12])):
        step = part.float().abs().amax(-1, keepdim=True) / (2 ** (bits - 1) - 1)
        # half a step, and the rounding of the value to bf16
        assert bool(((got.float() - part.float()).abs() <= 0.501 * step + 2.0 ** -8 * part.float().abs()).all())
    o = binding.mpq_cache_attention(rows[:, :8], table, lens, blk.cache, blk.codes, blk.scales)
    ol = binding.mpq_mx_layout(3, 8 * blk.dim)
    want = binding.mpq_mx_linear(binding.mpq_mx_quantize(o.view(3, -1), ol), ol, blk.w_out,
                                 blk.out_layout, dtype=blk.dtype)
    assert torch.equal(y, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = blk.step(x, slots, table, lens).clone()
    side.synchronize()
    assert torch.equal(z, y)
    cap = blk.capture(3, 3)
    for _ in range(2):
        cap.x.copy_(x)
        cap.slots.copy_(slots)
        cap.table.copy_(table)
        cap.lens.copy_(lens)
        assert torch.equal(cap.replay(), y)
        cap.lens.zero_()                      # nothing to attend to: zeros all the way
        assert not cap.replay().any()


def test_step_against_plain_arithmetic(gpu):
    """The block on the values its few-bit forms stand for, in fp64: the outputs agree to within the
    4-bit grid of the attended values (a relative step of 1/4 at most, 2^-2 / sqrt(12) of it rms)."""
    blk, gen = block()
    table, lens, slots = filled(blk, gen, [33, 20])
    x = torch.randn(2, blk.d, generator=gen, device=DEV).to(blk.dtype)
    y = blk.step(x, slots, table, lens).double()
    deq = lambda p, lay: binding.mpq_mx_dequantize(p, lay).double()
    wq, wo = deq(blk.w_qkv, blk.qkv_layout), deq(blk.w_out, blk.out_layout)
    xl = binding.mpq_mx_layout(2, blk.d)
    qkv = deq(binding.mpq_mx_quantize(x, xl), xl) @ wq.T
    q = qkv[:, :8 * 64].view(2, 8, 64)
    o = torch.zeros(2, 8, 64, dtype=torch.float64, device=DEV)
    for b, n in enumerate((33, 20)):
        t = torch.arange(n, device=DEV)
        at = table[b].long()[t // 16] * 16 + t % 16
        K, V = binding.mpq_cache_read(at, blk.cache, blk.codes, blk.scales, dtype=torch.float32)
        for h in range(8):
            p = torch.softmax(K[:, h // 4].double() @ q[b, h] / 8, 0)
            o[b, h] = p @ V[:, h // 4].double()
    want = o.view(2, -1) @ wo.T
    assert float((y - want).norm() / want.norm()) <= 0.25


def test_refusals(gpu):
    with pytest.raises(ValueError):
        FewBitAttention(torch.zeros(100, 64, device=DEV), torch.zeros(64, 128, device=DEV), 2, 1, 64, 4)
    blk, _ = block()
    with pytest.raises(ValueError):
        blk.step(torch.zeros(2, 100, device=DEV, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64,
                 device=DEV), torch.zeros(2, 1, dtype=torch.int32, device=DEV),
                 torch.ones(2, dtype=torch.int32, device=DEV))
