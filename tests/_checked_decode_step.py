"""The kernels of 4-bit integer weights, rotation and page tables on small seeded inputs, for
tests/test_gpu_checked_decode_step.py: run as a script (``MPQ_LIBRARY=<checked .so> python
tests/_checked_decode_step.py out.npz``) it saves the outputs."""
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
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    keep = lambda key, t: out.__setitem__(key, t.float().cpu().numpy())
    # weights: every group, types, whole and ragged rows, one tile a CTA and four
    for i, (rows, d, dtype) in enumerate(((3, 33, torch.float32), (130, 300, torch.float16), (200, 1096, torch.bfloat16),
                                          (5000, 2056, torch.bfloat16))):
        for group in (32, 64, 128):
            lay = binding.mpq_g4_layout(rows, d, group, i % 2 == 0)
            p = binding.mpq_g4_quantize(rand(rows, d).to(dtype), lay)
            keep(f"packed_{rows}_{group}", p)
            keep(f"values_{rows}_{group}", binding.mpq_g4_dequantize(p, lay, dtype=dtype))
    # the layer: one, two and four times eight tokens, tiles with K whole and split, CTA pairs, odd rows of x
    for T, C, d, group, dtype in ((1, 200, 4096, 128, torch.bfloat16), (13, 77, 333, 32, torch.float16),
                                  (40, 300, 1000, 64, torch.bfloat16), (150, 260, 4096, 32, torch.float16),
                                  (300, 14001, 264, 128, torch.bfloat16), (900, 4098, 515, 64, torch.bfloat16)):
        lay = binding.mpq_g4_layout(C, d, group, T % 2 == 0)
        w = binding.mpq_g4_quantize(rand(C, d), lay)
        for out_type in (torch.float32, dtype):
            keep(f"linear_{T}_{out_type}", binding.mpq_g4_linear(rand(T, d).to(dtype), w, lay, bias=rand(C), dtype=out_type))
    # rotation: rows of one warp and more, both pairings, rows off the 16-byte boundary
    for T, hq, h, dim, rot, neighbours in ((5, 4, 2, 64, 64, False), (70, 40, 8, 128, 64, True), (3, 5, 5, 50, 26, False),
                                           (300, 1, 1, 80, 80, False)):
        for dtype in (torch.float32, torch.bfloat16):
            rows = rand(T, hq + h, dim).to(dtype)
            turns = binding.mpq_rotation(10000.0 ** (-np.arange(0, rot, 2) / rot), DEV)
            pos = torch.arange(T, device=DEV, dtype=torch.int32) * 77
            q, k = rows.split((hq, h), 1)
            yq, yk = binding.mpq_rotate(q, k, pos, turns, norm=True, q_weight=rand(dim), neighbours=neighbours)
            keep(f"q_{T}_{dtype}", yq)
            keep(f"k_{T}_{dtype}", yk)
    # pages: room for all and for some, cut back
    for B, cols, spare in ((1, 3, 4), (40, 9, 60), (1500, 5, 3000)):
        lens = torch.randint(0, 20, (B,), generator=gen, device=DEV, dtype=torch.int32)
        table = torch.arange(B * cols, device=DEV, dtype=torch.int32).view(B, cols).contiguous()
        pool, count = torch.arange(spare, device=DEV, dtype=torch.int32) + B * cols, i32([spare, 0])
        add = torch.randint(0, 40, (B,), generator=gen, device=DEV, dtype=torch.int32)
        got = binding.mpq_pages_extend(add, lens, table, pool, count, 16, int(add.sum()) + 5)
        binding.mpq_pages_trim(lens // 2, lens, table, pool, count, 16)
        for name, t in zip(("slots", "positions", "taken", "lens", "table", "pool", "count"),
                           (*got, lens, table, pool, count)):
            keep(f"{name}_{B}", t)
    torch.cuda.synchronize()
    out["flags"] = np.array([binding.mpq_device_status()], dtype=np.int64)
    return out


if __name__ == "__main__":
    np.savez(sys.argv[1], build_options=np.array([binding.mpq_build_options()]), **outputs())
