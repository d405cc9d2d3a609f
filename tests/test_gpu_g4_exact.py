"""The linear layer with the values of 4-bit integer weights themselves (exact=True), s (q - z) in 64 bits.

Where every product and every partial sum, in whatever order, is a whole number of places that fp32 holds, outputs
have to be the reference's bit for bit: x of -1, 0 and 1, a row's scales m 2^e with m of 8 bits and one e, and so few
x other than 0 that their number times 15 * 255, the largest whole number of a weight, stays below 2^24.  A weight that
is rounded (to 8 or 11 bits), left out or taken twice shows there.

Elsewhere the bound: a weight is one or two terms, exact, whose magnitudes add up to (1 + 2^-8) |w| at most, and each
fp32 addition of the sum -- 2 d products (few tokens: d products, and a product with the scale and an addition for each
group), up to 16 where CTAs' and warps' sums are joined -- is off by at most one unit in the last place of a partial
sum, which the sum of magnitudes bounds: (2 d + d / 16 + 16) 2^-23 (1 + 2^-8) sum_j |x_j w_j| (+ the bias's addition, 2^-23
(|y| + |bias|)); the output's rounding adds 2^-24, 2^-11 or 2^-8 of |y| (fp32, fp16, bf16; fp16 also 2^-25
absolutely, and infinities past its range)."""
import numpy as np
import pytest
import torch

import _decode_step as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
# one token and a few; up to 128 tokens a tile, K whole and split over 2, 4 and 8 CTAs; up to 256, K whole and split; CTA pairs
SHAPES = [(1, 1, 1), (1, 300, 4096), (5, 77, 333), (9, 129, 1000), (20, 40, 333), (75, 520, 4097), (300, 203, 600),
          (513, 3001, 1000), (200, 64, 2560), (75, 4096, 11008), (250, 2000, 11001), (256, 4096, 4096), (700, 4000, 300),
          (1100, 5003, 333), (2100, 9001, 257), (1500, 9000, 140), (2300, 6001, 1100)]


def packed_matrix(gen, C, d, group, zeros, exponents, most=256):
    """(layout, packed buffer, values in 64 bits): every code, every zero point, scales m 2^e with m from 128 to most - 1 and
    an e a row; made on the device, where elements past the rows' ends have the value 0."""
    lay = binding.mpq_g4_layout(C, d, group, zeros)
    rt, kt, n = lay.row_tiles, lay.k_tiles, 128 // group
    rnd = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device=DEV)
    rows, wide = rt * 16, kt * 128
    q, m = rnd(0, 16, rows, wide), rnd(128, most, rows, kt * n)
    z = rnd(0, 16, rows, kt * n) if zeros else torch.full((rows, kt * n), 8, device=DEV)
    e = torch.zeros(rows, dtype=torch.float64, device=DEV)
    e[:C] = exponents
    s = torch.ldexp(m.double(), e[:, None]).bfloat16().double()          # (ldexp is off in the last of 53 bits)
    s[C:] = 0
    of = torch.arange(wide, device=DEV) // group
    q = torch.where(torch.arange(wide, device=DEV) < d, q, z[:, of])
    values = ((q - z[:, of]) * s[:, of])[:C, :d]
    w = q.view(rt, 16, kt, 4, 4, 8).permute(0, 2, 1, 4, 3, 5)             # word 4 i + m: elements 32 m + 8 i ..
    at = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=DEV)
    w = (w << at).sum(5)
    w = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32).reshape(rt, kt, -1).view(torch.uint8)
    per = lambda t: t.view(rt, 16, kt, n).permute(0, 2, 1, 3).reshape(rt, kt, -1).contiguous()
    parts = [w, per(s.bfloat16()).view(torch.uint8)] + ([per(z.to(torch.uint8))] if zeros else [])
    return lay, torch.cat(parts, 2).flatten().contiguous(), values


def ones(gen, T, d, dtype):
    """Rows of -1, 0 and 1, of which 4,096 at most are not 0."""
    x = torch.randint(0, 2, (T, d), generator=gen, device=DEV) * 2 - 1
    if d > 4096:
        x = x * (torch.rand(T, d, generator=gen, device=DEV).argsort(1) < 4096)
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("T,C,d", SHAPES)
@pytest.mark.parametrize("group,zeros,dtype", [(32, True, "bf16"), (64, False, "bf16"), (128, True, "fp16"),
                                               (32, False, "fp16")])
def test_whole_sums_bit_for_bit(gpu, T, C, d, group, zeros, dtype):
    """fp16: rows of scales far below and above fp16's range too."""
    gen = torch.Generator(device=DEV).manual_seed(T + C + d)
    lay, packed, w = packed_matrix(gen, C, d, group, zeros,
                                   torch.randint(-100, 90, (C,), generator=gen, device=DEV).double())
    x = ones(gen, T, d, dtype)
    want = (x.double() @ w.T).float()
    assert torch.equal(binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=True), want)
    assert binding.mpq_device_status() == 0


def layer(T, C, d, group, zeros, dtype, out, bias, seed, pad=0, shift=0):
    """(call, exact outputs, bounds) of a layer; rows of x `pad` elements apart from `shift` on, NaN between."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    x = (rand(T, d) * torch.exp(rand(T, 1))).to(TYPES[dtype])
    lay = binding.mpq_g4_layout(C, d, group, zeros)
    packed = binding.mpq_g4_quantize(0.05 * rand(C, d) * torch.exp(rand(C, 1)) + (0.02 if zeros else 0.0), lay)
    flat = torch.full((shift + T * (d + pad) + 8,), float("nan"), dtype=TYPES[dtype], device=DEV)
    rows = flat[shift:shift + T * (d + pad)].view(T, d + pad)[:, :d]
    rows.copy_(x)
    b = rand(C) if bias else None
    w = binding.mpq_g4_dequantize(packed, lay).double()                  # (12 bits: exact in fp32)
    return lambda **k: binding.mpq_g4_linear(rows, packed, lay, bias=b, exact=True, **(k or dict(dtype=TYPES[out]))), \
        *bounds(x, w, b, d, out)


def bounds(x, w, b, d, out):
    want = x.double() @ w.T
    tol = (2 * d + d / 16 + 16) * 2.0 ** -23 * (1 + 2.0 ** -8) * (x.double().abs() @ w.abs().T)
    if b is not None:
        want = want + b.double()
        tol = tol + 2.0 ** -23 * (want.abs() + b.double().abs())
    return want, tol + UNIT[out] * (want.abs() + tol) + (2.0 ** -25 if out == "fp16" else 0.0)


def within(y, want, tol):
    most = torch.finfo(y.dtype).max
    y = y.double()
    over = want.abs() - tol > most * (1 + 2.0 ** -11)
    near = ((y - want).abs() <= tol) | (y.isinf() & (want.abs() + tol > most) & (y * want > 0))
    return bool((near & (~over | y.isinf())).all())


@pytest.mark.parametrize("T,C,d", SHAPES)
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
def test_linear(gpu, T, C, d, group, zeros):
    dtype, out = ("bf16", "fp16")[(T + C) % 2], list(TYPES)[(T + C + group // 32) % 3]
    call, want, tol = layer(T, C, d, group, zeros, dtype, out, (T + d) % 2 == 0, T + C + d)
    y = call()
    assert y.shape == (T, C) and y.dtype == TYPES[out]
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("T,C,d,pad,shift", [(1, 40, 131, 0, 1), (5, 100, 333, 0, 0), (12, 77, 320, 8, 1), (90, 200, 1027, 2, 0),
                                             (300, 260, 333, 5, 3), (1400, 9001, 133, 3, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_odd_rows_repeated_bits_and_the_rest_left(gpu, T, C, d, pad, shift, dtype):
    """Rows of x off the 16-byte boundary and apart; equal bits from call to call; nothing is written beside the outputs."""
    call, want, tol = layer(T, C, d, 64, True, dtype, dtype, False, T + C, pad, shift)
    y = call()
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
    for gap in (0, 3):
        buf = torch.full((T + 1, C + gap), 3.0, dtype=TYPES[dtype], device=DEV)
        for _ in range(2):
            call(Y=buf[:T, :C])
            assert torch.equal(buf[:T, :C], y)
        assert bool((buf[:, C:] == 3.0).all()) and bool((buf[T] == 3.0).all())


def test_bf16_is_as_good_as_its_output(gpu):
    """With bf16 outputs the error is the outputs' own rounding: that of the exact sums rounded once, within 1%."""
    for T, C, d in ((1, 4096, 4096), (75, 1024, 4096), (400, 1024, 2048)):
        call, want, _ = layer(T, C, d, 64, True, "bf16", "bf16", False, T)
        least = (want.float().bfloat16().double() - want).norm()
        assert float((call().double() - want).norm()) <= 1.01 * float(least)


@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_of_scales_of_every_size(gpu, T, dtype):
    """A row's scales over 60 powers of two: fp16's many tokens hold a scale to 2^-36 of the row's largest, whose weights
    are at most 15 times it."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    C, d = 150, 1024
    lay = binding.mpq_g4_layout(C, d, 32, True)
    q = torch.randint(0, 16, (C, d), generator=gen, device=DEV).cpu().numpy().astype(np.uint8)
    z = torch.randint(0, 16, (C, 32), generator=gen, device=DEV).cpu().numpy().astype(np.uint8)
    s = ref.bf16(np.exp2(np.random.default_rng(T).uniform(-60, 0, (C, 32)) + np.linspace(-40, 40, C)[:, None]))
    packed = torch.from_numpy(ref.g4_pack(q, z, s, True)).to(DEV)
    w = torch.from_numpy(ref.g4_values(q, z, s, d)).to(DEV)
    x = torch.randn(T, d, generator=gen, device=DEV).to(TYPES[dtype])
    want, tol = bounds(x, w, None, d, "fp32")
    if dtype == "fp16":
        most = torch.from_numpy(s.astype(np.float64).max(1)).to(DEV)
        tol = tol + 15 * 2.0 ** -36 * most * x.double().abs().sum(1, keepdim=True)
    y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=True)
    assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [5, 60, 130, 1500])
def test_nan_and_infinity(gpu, T, dtype):
    """A NaN of the inputs makes its row NaN, a NaN group of the weights its column, nothing else; an infinity's row is
    infinite or NaN.  Columns of zeros alone are 0."""
    C, d = 140, 512
    gen = torch.Generator(device=DEV).manual_seed(T)
    x, w = torch.randn(T, d, generator=gen, device=DEV).to(TYPES[dtype]), torch.randn(C, d, generator=gen, device=DEV)
    x[3, 400] = float("nan")
    w[137, 5] = float("nan")
    w[20] = 0
    lay = binding.mpq_g4_layout(C, d, 64, True)
    packed = binding.mpq_g4_quantize(w, lay)
    bad = torch.zeros(T, C, dtype=torch.bool, device=DEV)
    bad[3], bad[:, 137] = True, True
    y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=True)
    assert torch.equal(torch.isnan(y), bad) and bool((y[~bad[:, 20], 20] == 0).all())
    x[3, 400] = float("inf")
    y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32, exact=True)
    assert not bool(torch.isfinite(y[3]).any()) and torch.equal(torch.isfinite(y), ~bad)


@pytest.mark.parametrize("T", [1, 30, 400])
def test_streams_graphs_and_empty_calls(gpu, T):
    call, _, _ = layer(T, 200, 776, 64, True, "bf16", "bf16", True, T)
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
    lay, lay0 = binding.mpq_g4_layout(40, 64, 32), binding.mpq_g4_layout(0, 64, 32)
    p = binding.mpq_g4_quantize(torch.ones(40, 64, device=DEV), lay)
    x = torch.ones(T, 64, dtype=torch.float16, device=DEV)
    assert binding.mpq_g4_linear(x[:0], p, lay, exact=True).shape == (0, 40)
    assert binding.mpq_g4_linear(x, p[:0], lay0, exact=True).shape == (T, 0)


def test_refusals(gpu):
    x = torch.zeros(4, 64, device=DEV)
    lay = binding.mpq_g4_layout(4, 64, 32)
    p = binding.mpq_g4_quantize(x, lay)
    with pytest.raises(binding.MPQError):
        binding.mpq_g4_linear(x, p, lay, exact=True)                      # fp32 inputs
    with pytest.raises(ValueError):
        binding.mpq_g4_linear(x.half()[:, :32], p, lay, exact=True)
    with pytest.raises(ValueError):
        binding.mpq_g4_linear(x.half(), p[:100], lay, exact=True)
