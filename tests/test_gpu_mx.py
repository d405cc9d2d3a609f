"""Microscaled 4-bit floats on the GPU: codes and scales bit for bit against the definition in 64 bits,
the values they stand for, and the linear layer against 64-bit sums of the same values.

The linear layer's bound: products are exact, and each of the d fp32 additions of a sum is off by at
most one unit in the last place of a partial sum, which the sum of magnitudes bounds, so
|y - exact| <= (d + 1) 2^-23 sum_j |x_j w_j| (+ the bias's addition, 2^-23 (|y| + |bias|)), and the
output's rounding adds 2^-24, 2^-11 or 2^-8 of |y| (fp32, fp16, bf16; fp16 also 2^-25 absolutely, and
infinities past its range)."""
import numpy as np
import pytest
import torch

import _serving as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def inputs(rows, d, seed, dtype="fp32"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, d)) * np.exp(rng.uniform(-3, 3, (rows, 1)))
    x[rng.random((rows, d)) < 0.02] *= 30
    x[rng.random((rows, d)) < 0.05] = 0
    return torch.from_numpy(x).to(TYPES[dtype])


def as64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 32), (3, 33), (2, 127), (129, 100), (5, 4096),
                                    (257, 130), (40, 2176), (1, 20001)])
def test_quantize_bits(gpu, rows, d, dtype):
    x = inputs(rows, d, rows * 7 + d, dtype)
    lay = binding.mpq_mx_layout(rows, d)
    packed = torch.full((lay.bytes,), 0xEE, dtype=torch.uint8, device=DEV)
    binding.mpq_mx_quantize(x.to(DEV), lay, packed)
    codes, exps = ref.mx_encode(as64(x))
    c, e, c_pad, e_all = ref.mx_unpack(packed.cpu().numpy(), rows, d)
    assert np.array_equal(c, codes) and np.array_equal(e, exps)
    assert not c_pad.any() and not e_all[:, exps.shape[1]:].any()
    # the scale bytes of the last row tile's missing rows
    full = packed.cpu().numpy()[lay.off_scales:].reshape(lay.row_tiles, lay.k_tiles, 32, 4, 4)
    full = full.transpose(0, 3, 2, 1, 4).reshape(lay.row_tiles * 128, -1)
    assert not full[rows:].any()
    # the values, in every type (fp16 overflows and underflows as a rounding would)
    for name, t in TYPES.items():
        got = binding.mpq_mx_dequantize(packed, lay, dtype=t)
        want = torch.from_numpy(ref.mx_decode(codes, exps)).to(torch.float32).to(t)
        assert torch.equal(got.cpu(), want), name


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,d", [(1, 716), (300, 230), (5, 1025), (129, 127), (2, 9525), (700, 31)])
def test_odd_rows_there_and_back(gpu, rows, d, dtype):
    """Rows off the 16-byte boundary: the bits of the same rows laid out on it, both ways."""
    x = inputs(rows, d, rows + d, dtype).to(DEV)
    wide = torch.zeros((rows, (d + 15) // 16 * 16 + 16), dtype=TYPES[dtype], device=DEV)
    wide[:, :d] = x
    lay = binding.mpq_mx_layout(rows, d)
    odd, even = binding.mpq_mx_quantize(x, lay), binding.mpq_mx_quantize(wide[:, :d], lay)
    assert torch.equal(odd, even)
    y = binding.mpq_mx_dequantize(odd, lay, dtype=TYPES[dtype])
    wide.fill_(7)
    binding.mpq_mx_dequantize(odd, lay, Y=wide[:, :d])
    assert torch.equal(torch.nan_to_num(wide[:, :d]), torch.nan_to_num(y)) and bool((wide[:, d:] == 7).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (0, 3)])
def test_quantize_strided_rows(gpu, dtype, pad, shift):
    """Rows further apart than d, bases off the 16-byte boundary."""
    rows, d = 70, 160
    x = inputs(rows, d, 5, dtype)
    buf = torch.full((shift + rows * (d + pad),), float("nan"), dtype=TYPES[dtype], device=DEV)
    view = buf[shift:].view(rows, d + pad)[:, :d]
    view.copy_(x)
    lay = binding.mpq_mx_layout(rows, d)
    assert torch.equal(binding.mpq_mx_quantize(view, lay), binding.mpq_mx_quantize(x.to(DEV), lay))
    out = torch.full_like(buf, 7.0)
    binding.mpq_mx_dequantize(binding.mpq_mx_quantize(view, lay), lay,
                              Y=out[shift:].view(rows, d + pad)[:, :d])
    want = binding.mpq_mx_dequantize(binding.mpq_mx_quantize(x.to(DEV), lay), lay, dtype=TYPES[dtype])
    got = out[shift:].view(rows, d + pad)
    assert torch.equal(got[:, :d], want)
    assert bool((got[:, d:] == 7.0).all()) and bool((out[:shift] == 7.0).all())


def test_quantize_special_values(gpu):
    """Ties at every midpoint, saturation, blocks of zeros, subnormals, the largest floats, NaN and
    infinities (whose block alone reads NaN)."""
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = []
    for e in (-140, -126, -30, 0, 20, 120, 125):
        r = np.zeros(64)
        r[:7], r[7:14] = mids, -mids
        r[14], r[15], r[16] = 4.0, 6.5, np.float32(7.9999995)
        r[32:39] = np.nextafter(mids.astype(np.float32), np.float32(9))
        r[39:46] = np.nextafter(mids.astype(np.float32), np.float32(0))
        r[46] = 4.0
        rows.append(np.ldexp(r, e))
    z = np.zeros(64)
    z[3] = -0.0
    rows.append(z)
    sub = np.zeros(64)
    sub[0], sub[1], sub[40] = 2.0 ** -149, -3 * 2.0 ** -149, 2.0 ** -127
    rows.append(sub)
    for bad in (np.nan, np.inf, -np.inf):
        r = np.linspace(-3, 3, 64)
        r[37] = bad
        rows.append(r)
    big = np.full(64, np.finfo(np.float32).max)
    big[1::2] = -1.0
    rows.append(big)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[~np.isfinite(x) & np.isfinite(np.array(rows))] = 0
    lay = binding.mpq_mx_layout(*x.shape)
    packed = binding.mpq_mx_quantize(torch.from_numpy(x).to(DEV), lay)
    codes, exps = ref.mx_encode(x)
    c, e, _, _ = ref.mx_unpack(packed.cpu().numpy(), *x.shape)
    assert np.array_equal(c, codes) and np.array_equal(e, exps)
    got = binding.mpq_mx_dequantize(packed, lay).cpu().numpy()
    want = ref.mx_decode(codes, exps).astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)


def test_dequantize_every_scale(gpu):
    """All 256 scale bytes with all 16 codes, among them those the quantiser never writes."""
    codes = np.tile(np.arange(16, dtype=np.uint8), (256, 2))
    exps = np.arange(256, dtype=np.uint8)[:, None]
    lay = binding.mpq_mx_layout(256, 32)
    packed = torch.from_numpy(ref.mx_pack(codes, exps)).to(DEV)
    with np.errstate(over="ignore"):
        want = ref.mx_decode(codes, exps).astype(np.float32)
    for t in TYPES.values():
        got = binding.mpq_mx_dequantize(packed, lay, dtype=t).cpu()
        assert torch.equal(torch.nan_to_num(got, nan=-7.0),
                           torch.nan_to_num(torch.from_numpy(want).to(t), nan=-7.0))


def linear(T, C, d, dtype, bias, seed):
    x, w = inputs(T, d, seed), 0.05 * inputs(C, d, seed + 1)
    xl, wl = binding.mpq_mx_layout(T, d), binding.mpq_mx_layout(C, d)
    xp, wp = binding.mpq_mx_quantize(x.to(DEV), xl), binding.mpq_mx_quantize(w.to(DEV), wl)
    b = torch.randn(C, generator=torch.Generator().manual_seed(seed)) if bias else None
    y = binding.mpq_mx_linear(xp, xl, wp, wl, bias=None if b is None else b.to(DEV),
                              dtype=TYPES[dtype])
    xv = torch.from_numpy(ref.mx_decode(*ref.mx_encode(as64(x)))).to(DEV)
    wv = torch.from_numpy(ref.mx_decode(*ref.mx_encode(as64(w)))).to(DEV)
    want, mag = xv @ wv.T, xv.abs() @ wv.abs().T
    tol = (d + 1) * 2.0 ** -23 * mag
    if b is not None:
        want = want + b.to(DEV).double()
        tol = tol + 2.0 ** -23 * (want.abs() + b.to(DEV).double().abs())
    tol = tol + UNIT[dtype] * (want.abs() + tol) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    return y, want, tol, (xp, xl, wp, wl)


def within(y, want, tol):
    """Every output within its bound; past fp16's largest number, the infinity it rounds to."""
    y, most = y.double(), torch.finfo(y.dtype).max
    over = want.abs() - tol > most * (1 + 2.0 ** -11)
    near = ((y - want).abs() <= tol) | (y.isinf() & (want.abs() + tol > most) & (y * want > 0))
    return bool((near & (~over | y.isinf())).all())


@pytest.mark.parametrize("T,C,d", [
    (1, 1, 1), (1, 128, 32), (1, 300, 4096), (15, 129, 257), (16, 127, 128), (17, 640, 1000),
    (63, 256, 384), (64, 256, 8192), (65, 130, 512), (128, 128, 256), (129, 384, 640),
    (200, 200, 2176), (255, 100, 96), (256, 256, 1024), (257, 129, 129), (700, 300, 770),
    (3, 20000, 130), (1030, 1030, 300), (1600, 1300, 300), (513, 3001, 1000), (5000, 300, 129),
    (2100, 2050, 512)])
def test_linear(gpu, T, C, d):
    dtype = list(TYPES)[(T + C) % 3]
    y, want, tol, _ = linear(T, C, d, dtype, (T + d) % 2 == 0, T + C + d)
    assert y.shape == (T, C) and y.dtype == TYPES[dtype]
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,C,d", [
    (33, 500, 64), (100, 96, 200), (200, 64, 2560), (330, 203, 700), (90, 4000, 100),
    (1000, 260, 1536), (2000, 61, 90), (150, 2052, 2048), (193, 5896, 2560), (200, 9000, 600),
    (352, 8136, 448), (700, 3080, 515)])
def test_linear_token_tiles(gpu, T, C, d, dtype):
    """Tiles of 32 to 256 tokens, some starting inside a block of 128 tokens' scales, K whole or split;
    channels by fours and one by one; the pairs' form with a last run of eight channels."""
    y, want, tol, _ = linear(T, C, d, dtype, C % 8 == 0, T + C + d)
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("T", [1, 40, 300])
def test_linear_fp32_outputs(gpu, T):
    y, want, tol, packed = linear(T, 260, 1536, "fp32", True, T)
    assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("T,C,d", [(1, 256, 4096), (30, 300, 8000), (300, 200, 600),
                                   (1600, 1304, 300), (1600, 1301, 300)])
def test_linear_repeats_bits_and_leaves_the_rest(gpu, T, C, d):
    """Equal bits from call to call; an output with rows further apart is written between them
    nowhere; nothing is written past either."""
    y, _, _, (xp, xl, wp, wl) = linear(T, C, d, "bf16", False, 11)
    buf = torch.full((T + 1, C + 5), 3.0, dtype=torch.bfloat16, device=DEV)
    for _ in range(3):
        binding.mpq_mx_linear(xp, xl, wp, wl, Y=buf[:T, :C])
        assert torch.equal(buf[:T, :C], y)
    assert bool((buf[:, C:] == 3.0).all()) and bool((buf[T] == 3.0).all())


@pytest.mark.parametrize("T", [5, 130, 9800])
def test_linear_nan_blocks(gpu, T):
    """A NaN block of the inputs makes its row NaN, one of the weights its column, nothing else."""
    C, d = 140, 512
    x, w = inputs(T, d, 1), inputs(C, d, 2)
    x[3, 400] = float("inf")
    w[137, 5] = float("nan")
    xl, wl = binding.mpq_mx_layout(T, d), binding.mpq_mx_layout(C, d)
    y = binding.mpq_mx_linear(binding.mpq_mx_quantize(x.to(DEV), xl), xl,
                              binding.mpq_mx_quantize(w.to(DEV), wl), wl, dtype=torch.float32)
    bad = torch.zeros(T, C, dtype=torch.bool, device=DEV)
    bad[3], bad[:, 137] = True, True
    assert torch.equal(torch.isnan(y), bad)


def test_empty_and_streams(gpu):
    lay0 = binding.mpq_mx_layout(0, 64)
    lay = binding.mpq_mx_layout(4, 64)
    p0 = binding.mpq_mx_quantize(torch.empty(0, 64, device=DEV), lay0)
    x = inputs(4, 64, 3).to(DEV)
    p = binding.mpq_mx_quantize(x, lay)
    assert binding.mpq_mx_linear(p0, lay0, p, lay).shape == (0, 4)
    assert binding.mpq_mx_linear(p, lay, p0, lay0).shape == (4, 0)
    want = binding.mpq_mx_linear(p, lay, p, lay)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.mpq_mx_linear(binding.mpq_mx_quantize(x, lay), lay, p, lay)
    side.synchronize()
    assert torch.equal(got, want)


def test_chain_of_dependent_calls(gpu):
    """Calls that follow one another on a stream, each reading what the one before has written."""
    d = 768
    lay = binding.mpq_mx_layout(40, d)
    wl = binding.mpq_mx_layout(d, d)
    x = inputs(40, d, 9).to(DEV)
    w = binding.mpq_mx_quantize((0.04 * inputs(d, d, 10)).to(DEV), wl)
    step = lambda y: binding.mpq_mx_linear(binding.mpq_mx_quantize(y, lay), lay, w, wl)
    want = x
    for _ in range(4):
        want = step(want)
        torch.cuda.synchronize()
    for _ in range(5):
        y = x
        for _ in range(4):
            y = step(y)
        assert torch.equal(y, want)


@pytest.mark.parametrize("T,C,d", [(4, 300, 512), (4, 300, 8192), (352, 8136, 448)])
def test_linear_withheld_copies_time_out(gpu, T, C, d):
    """With the test hook on, the kernel's waits run out with nothing in flight: the status says so, and the
    same call is right again after (K whole, K split over a cluster, CTA pairs)."""
    good, _, _, (xp, xl, wp, wl) = linear(T, C, d, "bf16", False, 3)
    assert binding.mpq_device_status() == 0
    try:
        binding.mpq_set_wait_limit(1 << 18)
        binding.mpq_test_withhold_copies(True)
        binding.mpq_mx_linear(xp, xl, wp, wl)
        flags = binding.mpq_device_status()
    finally:
        binding.mpq_test_withhold_copies(False)
        binding.mpq_set_wait_limit(0)
    assert flags == binding.MPQ_TIMEOUT_MX
    assert torch.equal(binding.mpq_mx_linear(xp, xl, wp, wl), good)
    assert binding.mpq_device_status() == 0


def test_linear_keeps_a_temporary_bias(gpu):
    """A bias that nothing but the call refers to is not overwritten by the output allocated in it."""
    T, C = 1, 600
    lay, wl = binding.mpq_mx_layout(T, 64), binding.mpq_mx_layout(C, 64)
    x = binding.mpq_mx_quantize(torch.zeros(T, 64, device=DEV), lay)
    w = binding.mpq_mx_quantize(torch.zeros(C, 64, device=DEV), wl)
    for i in range(20):
        y = binding.mpq_mx_linear(x, lay, w, wl, bias=torch.full((C,), float(i), device=DEV),
                                  dtype=torch.float32)
        assert bool((y == i).all())


def test_refusals(gpu):
    x = torch.zeros(4, 64, device=DEV)
    lay = binding.mpq_mx_layout(4, 64)
    p = binding.mpq_mx_quantize(x, lay)
    with pytest.raises(TypeError):
        binding.mpq_mx_quantize(x.int(), lay)
    with pytest.raises(ValueError):
        binding.mpq_mx_quantize(x.cpu(), lay)
    with pytest.raises(ValueError):
        binding.mpq_mx_quantize(x[:, :32], lay)
    with pytest.raises(ValueError):
        binding.mpq_mx_quantize(torch.zeros(64, 4, device=DEV).T, lay)
    with pytest.raises(ValueError):
        binding.mpq_mx_dequantize(p[:10], lay)
    with pytest.raises(binding.MPQError):
        binding.mpq_mx_linear(p, lay, p, binding.mpq_mx_layout(4, 32))
    with pytest.raises(TypeError):
        binding.mpq_mx_linear(p, lay, p, lay, bias=torch.zeros(4, device=DEV, dtype=torch.float16))
    with pytest.raises(binding.MPQError):
        binding.mpq_mx_layout(4, 0)
