"""The forms of the 4-bit integer layer, each asked for by mpq_test_g4_form; run as a script
(``MPQ_LIBRARY=<checked .so> python tests/_g4_forms.py out.npz``) it saves the forms' outputs on small seeded
inputs, for tests/test_gpu_g4_forms.py."""
import contextlib
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2002_09049_gb300 import binding  # noqa: E402

DEV = "cuda:0"
FEW, PAIRS = (binding.MPQ_G4_FEW, 0, 1), (binding.MPQ_G4_PAIRS, 0, 1)
TILES = [(binding.MPQ_G4_TILES, n, s) for n, s in ((32, 1), (48, 8), (80, 4), (128, 1), (128, 2), (144, 1), (192, 2),
                                                   (256, 1), (256, 4), (256, 8))]
FORMS = [FEW, *TILES, PAIRS]


@contextlib.contextmanager
def form(f):
    binding.mpq_test_g4_form(*f)
    try:
        yield
    finally:
        binding.mpq_test_g4_form()


def least(f, d):
    """A row length like d that the form takes: two packed tiles or more for each CTA that shares K."""
    return d if f[2] == 1 else max(d, 256 * f[2] + d % 128)


def outputs():
    out = {}
    gen = torch.Generator(device=DEV).manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    for i, f in enumerate(FORMS):
        for T, C, d in ((37, 130, 300), (300, 517, 1153)):
            dtype, d = (torch.bfloat16, torch.float16)[(i + T) % 2], least(f, d)
            lay = binding.mpq_g4_layout(C, d, (32, 64, 128)[i % 3], i % 2 == 0)
            w, x, b = binding.mpq_g4_quantize(rand(C, d), lay), rand(T, d).to(dtype), rand(C)
            with form(f):
                for exact in (False, True):
                    for kind in (torch.float32, dtype):
                        out[f"{f}_{T}_{exact}_{kind}"] = binding.mpq_g4_linear(
                            x, w, lay, bias=b, dtype=kind, exact=exact).float().cpu().numpy()
    torch.cuda.synchronize()
    out["flags"] = np.array([binding.mpq_device_status()], dtype=np.int64)
    return out


if __name__ == "__main__":
    np.savez(sys.argv[1], build_options=np.array([binding.mpq_build_options()]), **outputs())
