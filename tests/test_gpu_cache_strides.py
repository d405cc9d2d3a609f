"""Keys and values whose strides differ where there is nothing to stride over are one call like any other."""
import pytest
import torch

from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,heads", [(1, 3), (5, 1), (1, 1)])
def test_dimensions_of_one_entry(gpu, T, heads, dtype):
    dim = 64
    lay = binding.mpq_cache_layout(2, 16, heads, dim, 8)
    x = torch.randn(2, T, heads, dim, device=DEV).to(dtype)
    # the values: rows of their own places, as far apart as the keys' wherever there is a next one
    step = (heads * dim if T > 1 else 11 * dim, dim if heads > 1 else 5 * dim)
    V = torch.full((T * heads * dim + 16,), 7.0, device=DEV, dtype=dtype).as_strided((T, heads, dim), (*step, 1))
    V.copy_(x[1])
    K = x[0]
    assert K.stride() != V.stride()
    slots = torch.arange(T, device=DEV) + 3
    a, b = binding.mpq_cache_empty(lay, DEV), binding.mpq_cache_empty(lay, DEV)
    binding.mpq_cache_write(K, V, slots, lay, *a)
    binding.mpq_cache_write(K, V.clone(memory_format=torch.contiguous_format), slots, lay, *b)
    for u, v in zip(binding.mpq_cache_read(slots, lay, *a), binding.mpq_cache_read(slots, lay, *b)):
        assert torch.equal(u, v)


def test_strides_that_matter_are_still_compared(gpu):
    lay = binding.mpq_cache_layout(2, 16, 2, 64, 8)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    wide = torch.zeros(4, 3, 64, device=DEV)
    slots = torch.arange(4, device=DEV)
    with pytest.raises(ValueError, match="strides"):
        binding.mpq_cache_write(torch.zeros(4, 2, 64, device=DEV), wide[:, :2], slots, lay, codes, scales)
    with pytest.raises(ValueError, match="contiguous"):
        t = torch.zeros(4, 64, 2, device=DEV).transpose(1, 2)
        binding.mpq_cache_write(t, t, slots, lay, codes, scales)
