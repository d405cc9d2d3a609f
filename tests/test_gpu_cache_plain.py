"""The bytes that the cache holds are those of the same formula in PyTorch operations on the GPU, perf/operators.py's
plain form (its division of the row's largest by Qmax, a number, is there a product with the rounded reciprocal,
as include/mpq.h says of the scale), and their scales are within a unit in the last place of the quotient."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HERE = os.path.dirname(os.path.abspath(__file__))


def plain():
    spec = importlib.util.spec_from_file_location(
        "operators", os.path.join(os.path.dirname(HERE), "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [64, 256])
def test_bytes_are_the_plain_forms(gpu, dim, bits, dtype):
    T, heads, page = 3000, 2, 16
    gen = torch.Generator(device=DEV).manual_seed(dim + bits)
    kv = torch.randn(T, 2, heads, dim, generator=gen, device=DEV)
    kv = (kv * torch.exp(2 * torch.randn(T, 2, heads, 1, generator=gen, device=DEV))).to(dtype)
    lay = binding.mpq_cache_layout(-(-T // page), page, heads, dim, bits)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    slots = torch.arange(T, device=DEV)
    binding.mpq_cache_write(kv[:, 0], kv[:, 1], slots, lay, codes, scales)
    rows, s = plain()._cache_store(kv.float(), bits)
    at = (slots // page, slice(None), slice(None), slots % page)
    assert torch.equal(scales[at], s) and torch.equal(codes[at], rows)
    top = kv.float().abs().amax(-1).cpu().numpy()
    want = top / np.float32(2 ** (bits - 1) - 1)
    off = np.abs(scales[at].cpu().numpy().view(np.int32).astype(np.int64) - want.view(np.int32))
    assert off.max() <= 1
