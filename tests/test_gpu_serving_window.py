"""A step of the few-bit attention block with a window: its calls, bit for bit, in eager and captured form, and
other outputs than with a window one token wider."""
import pytest
import torch

from paper_2002_09049_gb300 import binding
from test_gpu_streams import batch, block, replayed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("window", [1, 16, 33])
def test_step_with_a_window(gpu, window, bits):
    blk, gen = block(bits)
    args = batch(blk, gen, 0, [60, 40, 64])
    x, slots, table, lens = args
    y = blk.step(*args, window=window).clone()
    xl = binding.mpq_mx_layout(3, blk.d)
    qkv = binding.mpq_mx_linear(binding.mpq_mx_quantize(x, xl), xl, blk.w_qkv, blk.qkv_layout, dtype=blk.dtype)
    ol = binding.mpq_mx_layout(3, 8 * 64)
    outs = []
    for w in (window, window + 1):
        o = binding.mpq_cache_attention(qkv.view(3, -1, 64)[:, :8], table, lens, blk.cache, blk.codes, blk.scales,
                                        window=w)
        outs.append(binding.mpq_mx_linear(binding.mpq_mx_quantize(o.view(3, -1), ol), ol, blk.w_out,
                                          blk.out_layout, dtype=blk.dtype))
    assert torch.equal(y, outs[0]) and not torch.equal(y, outs[1])
    assert torch.equal(replayed(blk.capture(3, 4, window), args), y)
