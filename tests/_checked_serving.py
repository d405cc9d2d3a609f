"""Every kernel of the few-bit serving calls on small seeded inputs, for tests/test_gpu_checked_serving.py:
run as a script (``MPQ_LIBRARY=<checked .so> python tests/_checked_serving.py out.npz``) it saves the
outputs, so that a test can compare a checked-build process with the normal build."""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2002_09049_gb300 import binding  # noqa: E402

DEV = "cuda:0"


def outputs():
    out = {}
    gen = torch.Generator(device=DEV).manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    keep = lambda key, t: out.__setitem__(key, t.float().cpu().numpy())
    # microscaled floats: every type, ragged rows; the linear layer's forms (a few tokens with K split and
    # not, one CTA's tiles, CTA pairs)
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        for rows, d in ((3, 33), (130, 300)):
            lay = binding.mpq_mx_layout(rows, d)
            p = binding.mpq_mx_quantize(rand(rows, d).to(dtype), lay)
            keep(f"mx_{dtype}_{rows}", binding.mpq_mx_dequantize(p, lay, dtype=dtype))
    for T, C, d, dtype in ((1, 200, 4096, torch.bfloat16), (40, 21000, 100, torch.float16),
                           (300, 130, 300, torch.float32), (1600, 1301, 300, torch.bfloat16)):
        xl, wl = binding.mpq_mx_layout(T, d), binding.mpq_mx_layout(C, d)
        y = binding.mpq_mx_linear(binding.mpq_mx_quantize(rand(T, d), xl), xl,
                                  binding.mpq_mx_quantize(rand(C, d), wl), wl, bias=rand(C),
                                  dtype=dtype)
        keep(f"linear_{T}", y)
    # the cache and its attention: widths, head groups, rows of one warp, of several, of several CTAs
    for dim, bits, heads, group, lens in ((64, 8, 2, 3, [5, 0, 70]), (128, 4, 1, 12, [900, 33]),
                                          (256, 8, 1, 2, [300, 1]), (128, 8, 1, 4, [9000])):
        need = [-(-n // 16) for n in lens]
        lay = binding.mpq_cache_layout(sum(need) + 1, 16, heads, dim, bits)
        codes, scales = binding.mpq_cache_empty(lay, DEV)
        codes.zero_()
        scales.zero_()
        T = sum(need) * 16
        kv = rand(2, T, heads, dim).to(torch.bfloat16)
        slots = torch.arange(T, device=DEV)
        binding.mpq_cache_write(kv[0], kv[1], slots, lay, codes, scales)
        K, V = binding.mpq_cache_read(slots[:50], lay, codes, scales, dtype=torch.float32)
        table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = torch.arange(at, at + n, device=DEV)
            at += n
        lse = torch.empty((len(lens), heads * group), device=DEV)
        o = binding.mpq_cache_attention(rand(len(lens), heads * group, dim).to(torch.bfloat16), table,
                                        torch.tensor(lens, dtype=torch.int32, device=DEV), lay, codes,
                                        scales, lse=lse)
        for name, t in dict(K=K, V=V, o=o, lse=lse).items():
            keep(f"{name}_{dim}_{bits}_{len(lens)}", t)
    torch.cuda.synchronize()
    out["flags"] = np.array([binding.mpq_device_status()], dtype=np.int64)
    return out


if __name__ == "__main__":
    np.savez(sys.argv[1], build_options=np.array([binding.mpq_build_options()]), **outputs())
