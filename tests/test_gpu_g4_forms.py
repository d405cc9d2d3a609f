"""Every form of the 4-bit integer layer -- a few tokens' kernel, tiles of up to 128 and up to 256 tokens with K whole and
split, CTA pairs -- against 64-bit references, whatever sizes would choose it: both calls (the weights' values
rounded to x's type, and exact), ragged ends, NaN, scales out of fp16's range, graphs, the checked build, the
timeout.

Whole sums are compared bit for bit, so that no term can be missing, double or rounded: test_gpu_g4_exact.py says why they
are exact in any order; the rounded call's scales are powers of two, whose values both types hold.  Random data's
bounds are those of test_gpu_g4_exact.py, with the values rounded to x's type (one term, less than its two) in
the rounded call."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import _decode_step as ref
import _g4_forms
from _g4_forms import DEV, FEW, FORMS, PAIRS, TILES, form, least
from test_gpu_g4_exact import TYPES, bounds, ones, packed_matrix, within
from paper_2002_09049_gb300 import _build, binding

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ids = lambda f: "-".join(map(str, f))


def matrix(gen, C, d, group, zeros, dtype, exact):
    if exact:
        return packed_matrix(gen, C, d, group, zeros, torch.randint(-100, 90, (C,), generator=gen, device=DEV).double())
    e = torch.randint(-16, -6, (C,), generator=gen, device=DEV).double()
    return packed_matrix(gen, C, d, group, zeros, e, 129)


@pytest.mark.parametrize("f", FORMS, ids=ids)
@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("T,C,d", [(1, 129, 128), (37, 300, 1000), (300, 700, 2113), (130, 129, 65), (523, 20001, 257),
                                   (90, 260, 11008)])
def test_whole_sums_bit_for_bit(gpu, f, exact, T, C, d):
    """(523 x 20,001: more tiles than CTAs are resident, in every form.)"""
    d = least(f, d)
    gen = torch.Generator(device=DEV).manual_seed(T + C + d)
    kinds = ((32, True, "bf16"), (64, False, "fp16"), (128, True, "fp16"), (128, False, "bf16"))
    for group, zeros, dtype in kinds[:2] if (T + d) % 2 else kinds[2:]:
        lay, packed, w = matrix(gen, C, d, group, zeros, dtype, exact)
        x = ones(gen, T, d, dtype)
        with form(f):
            y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=exact)
        assert torch.equal(y, (x.double() @ w.T).float())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("f", FORMS, ids=ids)
@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("T,C,d,gap,shift", [(300, 516, 1152, 0, 0), (261, 387, 1153, 3, 1), (70, 130, 520, 8, 4)])
def test_random(gpu, f, exact, T, C, d, gap, shift):
    """Every output type, with a bias, rows of x and Y apart and off their boundaries; equal bits twice, nothing beside the
    outputs written."""
    d = least(f, d)
    gen = torch.Generator(device=DEV).manual_seed(T)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    for dtype, group, zeros in (("bf16", 64, True), ("fp16", 32, False), ("fp16", 128, True)):
        lay = binding.mpq_g4_layout(C, d, group, zeros)
        packed, b = binding.mpq_g4_quantize(0.05 * rand(C, d) + (0.02 if zeros else 0), lay), rand(C)
        flat = torch.full((shift + T * (d + gap),), float("nan"), dtype=TYPES[dtype], device=DEV)
        x = flat[shift:].view(T, d + gap)[:, :d]
        x.copy_(rand(T, d))
        w = binding.mpq_g4_dequantize(packed, lay, dtype=torch.float32 if exact else TYPES[dtype]).double()
        for out in TYPES:
            want, tol = bounds(x, w, b, d, out)
            buf = torch.full((T + 1, C + gap), 3.0, dtype=TYPES[out], device=DEV)
            with form(f):
                y = binding.mpq_g4_linear(x, packed, lay, bias=b, dtype=TYPES[out], exact=exact)
                binding.mpq_g4_linear(x, packed, lay, bias=b, Y=buf[:T, :C], exact=exact)
            assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
            assert torch.equal(buf[:T, :C], y)
            assert bool((buf[:, C:] == 3.0).all()) and bool((buf[T] == 3.0).all())


@pytest.mark.parametrize("f", FORMS, ids=ids)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scales_of_every_size_and_nan(gpu, f, dtype):
    """The rounded call's values are those that the matrix stands for in x's type, subnormal, vanished and infinite ones
    among them (x is one row of the identity at a time); a NaN of the inputs makes its row NaN, a NaN scale its column."""
    d, T = least(f, 128), 290
    s = np.exp2(np.arange(-140, 126, dtype=np.float64)).astype(np.float32)
    s = ref.bf16(np.concatenate([s, s * 1.5078125, -s * 1.9921875]))[:, None].repeat(-(-d // 128) * 4, 1)
    rng = np.random.default_rng(1)
    q, z = rng.integers(0, 16, (len(s), s.shape[1] * 32)).astype(np.uint8), rng.integers(0, 16, s.shape).astype(np.uint8)
    q[:, d:], z[:, -(-d // 32):] = 8, 8
    lay = binding.mpq_g4_layout(len(s), d, 32, True)
    packed = torch.from_numpy(ref.g4_pack(q, z, s, True)).to(DEV)
    want = binding.mpq_g4_dequantize(packed, lay, dtype=TYPES[dtype])
    rows = torch.arange(T, device=DEV) % d
    x = torch.nn.functional.one_hot(rows, d).to(TYPES[dtype])
    finite = torch.isfinite(want).all(1)                            # (0 times infinity is NaN)
    with form(f):
        y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32)
    small = want.abs() < 2.0 ** -126                                # (fp32 sums may drop their subnormals)
    assert torch.equal(torch.where(small[finite][:, rows], 0.0, y[:, finite].T),
                       torch.where(small, torch.zeros_like(want), want)[finite][:, rows].float())
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(2)).to(TYPES[dtype])
    w = torch.randn(140, d, generator=torch.Generator().manual_seed(3))
    x[3, 40] = w[137, 5] = float("nan")
    lay = binding.mpq_g4_layout(140, d, 32, False)
    packed = binding.mpq_g4_quantize(w.to(DEV), lay)
    bad = torch.zeros(T, 140, dtype=torch.bool, device=DEV)
    bad[3], bad[:, 137] = True, True
    for exact in (False, True):
        with form(f):
            y = binding.mpq_g4_linear(x.to(DEV), packed, lay, dtype=torch.float32, exact=exact)
        assert torch.equal(torch.isnan(y), bad)


@pytest.mark.parametrize("f", FORMS, ids=ids)
def test_chain_and_its_graph(gpu, f):
    """Calls that follow one another on a stream, each reading what the one before has written, and their replay."""
    T, d = 270, least(f, 776)
    gen = torch.Generator(device=DEV).manual_seed(9)
    lay = binding.mpq_g4_layout(d, d, 64, True)
    w = binding.mpq_g4_quantize(torch.randn(d, d, generator=gen, device=DEV) / d ** 0.5, lay)
    x = torch.randn(T, d, generator=gen, device=DEV).bfloat16()

    def chain(after=lambda: None):
        y = x
        for i in range(4):
            y = binding.mpq_g4_linear(y, w, lay, exact=i % 2 == 1)
            after()
        return y
    with form(f):
        want = chain(torch.cuda.synchronize)
        assert bool(want.isfinite().all())
        for _ in range(5):
            assert torch.equal(chain(), want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = chain()
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)


def test_checked_build(gpu, tmp_path):
    """In the checked build no index check fails, and every output equals the normal build's, bit for bit."""
    out = tmp_path / "checked.npz"
    r = subprocess.run([sys.executable, os.path.join(HERE, "_g4_forms.py"), str(out)],
                       env=dict(os.environ, MPQ_LIBRARY=_build.build(checked=True)), capture_output=True, text=True,
                       timeout=900)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    with np.load(out) as z:
        checked = {k: z[k] for k in z.files}
    assert int(checked["build_options"][0]) & binding.MPQ_BUILD_CHECK_BOUNDS
    assert int(checked["flags"][0]) == 0
    normal = _g4_forms.outputs()
    assert int(normal["flags"][0]) == 0
    for key, want in normal.items():
        assert np.array_equal(checked[key], want, equal_nan=True), key


@pytest.mark.parametrize("f", [*TILES, PAIRS], ids=ids)
@pytest.mark.parametrize("exact", [False, True])
def test_withheld_copies_time_out(gpu, f, exact):
    """With the test hook on, the kernel's waits run out with nothing in flight: the status says so, and the same call is
    right again after."""
    d = least(f, 520)
    gen = torch.Generator(device=DEV).manual_seed(3)
    lay, packed, w = packed_matrix(gen, 700, d, 64, False, torch.zeros(700, dtype=torch.float64, device=DEV), 129)
    x = ones(gen, 600, d, "bf16")
    want = (x.double() @ w.T).float()
    with form(f):
        try:
            binding.mpq_set_wait_limit(1 << 18)
            binding.mpq_test_withhold_copies(True)
            binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=exact)
            flags = binding.mpq_device_status()
        finally:
            binding.mpq_test_withhold_copies(False)
            binding.mpq_set_wait_limit(0)
        assert flags == binding.MPQ_TIMEOUT_G4
        assert torch.equal(binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=exact), want)
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("f", [*TILES, PAIRS], ids=ids)
@pytest.mark.parametrize("T,d", [(40, 2100), (600, 2100), (300, 200)])
def test_withheld_weights_time_out(gpu, f, T, d):
    """With copies of x landed and the weights' withheld, the kernel ends as soon: its copies need no other role's work to
    be waited for, so no drain gives up."""
    d = least(f, d)
    gen = torch.Generator(device=DEV).manual_seed(4)
    lay, packed, w = packed_matrix(gen, 700, d, 64, False, torch.zeros(700, dtype=torch.float64, device=DEV), 129)
    x = ones(gen, T, d, "bf16")
    with form(f):
        try:
            binding.mpq_set_wait_limit(1 << 18)
            binding.mpq_test_withhold_copies(2)
            binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32)
            flags = binding.mpq_device_status()
        finally:
            binding.mpq_test_withhold_copies(0)
            binding.mpq_set_wait_limit(0)
        assert flags == binding.MPQ_TIMEOUT_G4
        assert torch.equal(binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32), (x.double() @ w.T).float())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("f", [(binding.MPQ_G4_TILES, 48, 8), (binding.MPQ_G4_TILES, 256, 2), PAIRS], ids=ids)
def test_beside_the_microscaled_layer(gpu, f):
    """The two layers whose clusters' CTAs allocate tensor memory, on two streams and one after another on one: each ends,
    with the result of the call made alone (an SM has no room for CTAs of both)."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    d, T = 4096, 48
    lay, xl, wl = binding.mpq_g4_layout(4096, d, 64), binding.mpq_mx_layout(T, d), binding.mpq_mx_layout(1500, d)
    g, w = binding.mpq_g4_quantize(rand(4096, d), lay), binding.mpq_mx_quantize(rand(1500, d), wl)
    x = rand(T, d).bfloat16()
    q = binding.mpq_mx_quantize(x, xl)
    one, two = lambda: binding.mpq_g4_linear(x, g, lay), lambda: binding.mpq_mx_linear(q, xl, w, wl)
    with form(f):
        y, v = one(), two()
        torch.cuda.synchronize()
        streams = torch.cuda.Stream(), torch.cuda.Stream()
        for _ in range(40):
            got = []
            for s, calls in zip(streams, ((one, two, one), (two, one, two))):
                with torch.cuda.stream(s):
                    got += [(c, c()) for c in calls]
            torch.cuda.synchronize()
            assert all(torch.equal(r, y if c is one else v) for c, r in got)
    assert binding.mpq_device_status() == 0


def test_a_form_that_a_call_cannot_take(gpu):
    lay = binding.mpq_g4_layout(16, 512, 64)
    p = binding.mpq_g4_quantize(torch.ones(16, 512, device=DEV), lay)
    with form((binding.MPQ_G4_TILES, 64, 4)), pytest.raises(binding.MPQError):
        binding.mpq_g4_linear(torch.ones(20, 512, device=DEV, dtype=torch.float16), p, lay)
    assert bool((binding.mpq_g4_linear(torch.ones(20, 512, device=DEV, dtype=torch.float16), p, lay) > 0).all())
