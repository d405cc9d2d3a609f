"""4-bit integer weights on the GPU: codes, zero points and scales bit for bit against the definition, the
values they stand for, and the linear layer against 64-bit sums of the same values.

The linear layer's bound: products of x and the weights' values in x's type are exact, and each fp32 addition of a
sum -- d products, up to 16 where CTAs' and warps' sums are joined -- is off by at most one unit in the last place of a
partial sum, which the sum of magnitudes bounds: |y - exact| <= (d + 16) 2^-23 sum_j |x_j w_j| (+ the bias's
addition, 2^-23 (|y| + |bias|)); the output's rounding adds 2^-24, 2^-11 or 2^-8 of |y| (fp32, fp16, bf16;
fp16 also 2^-25 absolutely, and infinities past its range)."""
import numpy as np
import pytest
import torch

import _decode_step as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
KINDS = [(g, z) for g in ref.GROUPS for z in (False, True)]


def inputs(rows, d, seed, dtype="fp32", shift=0.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, d)) * np.exp(rng.uniform(-3, 3, (rows, 1))) + shift
    x[rng.random((rows, d)) < 0.02] *= 30
    x[rng.random((rows, d)) < 0.05] = 0
    x[:, d // 2:d // 2 + 140][rows // 2:] = 0                     # whole groups of zeros
    return torch.from_numpy(x).to(TYPES[dtype])


def packed_of(q, z, s, zeros):
    return torch.from_numpy(ref.g4_pack(q, z, s, zeros))


@pytest.mark.parametrize("group,zeros", KINDS)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 33), (16, 128), (17, 129), (2, 700), (50, 384)])
def test_quantize_bits(gpu, rows, d, group, zeros):
    dtype = list(TYPES)[(rows + d + group) % 3]
    x = inputs(rows, d, rows * 7 + d, dtype, 0.4)
    lay = binding.mpq_g4_layout(rows, d, group, zeros)
    packed = torch.full((lay.bytes,), 0xEE, dtype=torch.uint8, device=DEV)
    binding.mpq_g4_quantize(x.to(DEV), lay, packed)
    q, z, s = ref.g4_encode(x.float().numpy(), group, zeros)
    assert torch.equal(packed.cpu(), packed_of(q, z, s, zeros))
    for t in TYPES.values():
        want = torch.from_numpy(ref.g4_values(q, z, s, d)).to(torch.float32).to(t)
        assert torch.equal(binding.mpq_g4_dequantize(packed, lay, dtype=t).cpu(), want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (0, 3)])
def test_quantize_strided_rows(gpu, dtype, pad, shift):
    """Rows further apart than d, bases off the 16-byte boundary; nothing is written between them."""
    rows, d = 70, 200
    x = inputs(rows, d, 5, dtype)
    buf = torch.full((shift + rows * (d + pad),), float("nan"), dtype=TYPES[dtype], device=DEV)
    view = buf[shift:].view(rows, d + pad)[:, :d]
    view.copy_(x)
    lay = binding.mpq_g4_layout(rows, d, 64, True)
    packed = binding.mpq_g4_quantize(view, lay)
    assert torch.equal(packed, binding.mpq_g4_quantize(x.to(DEV), lay))
    out = torch.full_like(buf, 7.0)
    binding.mpq_g4_dequantize(packed, lay, Y=out[shift:].view(rows, d + pad)[:, :d])
    got = out[shift:].view(rows, d + pad)
    assert torch.equal(got[:, :d], binding.mpq_g4_dequantize(packed, lay, dtype=TYPES[dtype]))
    assert bool((got[:, d:] == 7.0).all()) and bool((out[:shift] == 7.0).all())


@pytest.mark.parametrize("group,zeros", KINDS)
def test_quantize_special_values(gpu, group, zeros):
    """Quotients on and beside the borders between codes, subnormals, the largest floats, NaN and infinities
    (whose group alone reads NaN), one sign only."""
    rows = []
    for e in (-146, -133, -126, -101, -30, 0, 99, 125):
        mids = np.arange(-7.5, 8) / 8
        with np.errstate(over="ignore"):
            r = np.concatenate([mids, np.nextafter(mids.astype(np.float32), np.float32(9)),
                                np.nextafter(mids.astype(np.float32), np.float32(-9)), [7.0 / 8, -7.0 / 8]])
            rows.append(np.ldexp(np.resize(r, 128), e))
    for bad in (np.nan, np.inf, -np.inf):
        r = np.linspace(-3, 3, 128)
        r[37] = bad
        rows.append(r)
    big = np.full(128, np.finfo(np.float32).max)
    rows.append(big.copy())
    big[1::2] *= -1
    rows += [big, np.linspace(1, 2, 128), np.linspace(-2, -1, 128), np.zeros(128), np.full(128, -0.0)]
    x = np.array(rows).astype(np.float32)
    lay = binding.mpq_g4_layout(*x.shape, group, zeros)
    packed = binding.mpq_g4_quantize(torch.from_numpy(x).to(DEV), lay)
    q, z, s = ref.g4_encode(x, group, zeros)
    got = binding.mpq_g4_dequantize(packed, lay).cpu().numpy()
    assert np.array_equal(got, ref.g4_values(q, z, s, 128).astype(np.float32), equal_nan=True)
    finite = np.isfinite(s).all(1)                    # (which NaN a scale is, is not said)
    want = packed_of(q[finite], z[finite], s[finite], zeros)
    again = binding.mpq_g4_quantize(torch.from_numpy(x[finite]).to(DEV),
                                    binding.mpq_g4_layout(int(finite.sum()), 128, group, zeros))
    assert torch.equal(again.cpu(), want)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("group,zeros", KINDS)
def test_quantize_every_16_bit_float(gpu, group, zeros, dtype):
    """Every 16-bit float -- both zeros, subnormals, infinities, NaN -- in order and out of it, and ranges whose two
    ends both round away from zero: as the definition has them, and as the same floats in fp32."""
    bits = np.arange(65536, dtype=np.uint16)
    mixed = np.random.default_rng(9).permutation(bits)
    x = torch.from_numpy(np.concatenate([bits, mixed, mixed | 0x8000]).view(np.int16)).view(TYPES[dtype]).view(-1, 128)
    ends = torch.zeros(512, 128, dtype=TYPES[dtype])
    ends[:, ::2] = (1 + torch.arange(512) / 512)[:, None] * 5.5
    ends[:, 1::2] = -9.5
    x = torch.cat([x, ends])
    lay = binding.mpq_g4_layout(*x.shape, group, zeros)
    packed = binding.mpq_g4_quantize(x.to(DEV), lay)
    assert torch.equal(packed, binding.mpq_g4_quantize(x.float().to(DEV), lay))
    q, z, s = ref.g4_encode(x.float().numpy(), group, zeros)
    got = binding.mpq_g4_dequantize(packed, lay).cpu().numpy()
    with np.errstate(over="ignore", invalid="ignore"):
        want = ref.g4_values(q, z, s, 128).astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)
    wide = torch.empty(x.shape[0], 129, dtype=TYPES[dtype], device=DEV)[:, 1:]        # rows off the 16-byte boundary
    assert torch.equal(binding.mpq_g4_quantize(wide.copy_(x), lay), packed)
    many = x.view(16, -1).repeat(80, 1).to(DEV)                                       # several tiles a thread
    lay = binding.mpq_g4_layout(*many.shape, group, zeros)
    packed = binding.mpq_g4_quantize(many, lay)
    assert torch.equal(packed, binding.mpq_g4_quantize(many.float(), lay))
    assert torch.equal(packed.view(80, -1), packed[:packed.numel() // 80].expand(80, -1))
    assert torch.equal(binding.mpq_g4_dequantize(packed, lay)[:16].nan_to_num(7.0).cpu(),
                       torch.from_numpy(got).view(16, -1).nan_to_num(7.0))


@pytest.mark.parametrize("group,zeros", KINDS)
def test_every_code(gpu, group, zeros):
    """Buffers made elsewhere: every code with every zero point, scales of either sign."""
    d = 256
    q = np.resize(np.arange(16, dtype=np.uint8), (32, d))
    n = d // group
    z = (np.arange(32)[:, None] + np.arange(n)) % 16 if zeros else np.full((32, n), 8)
    s = ref.bf16(np.random.default_rng(2).standard_normal((32, n)).astype(np.float32))
    packed = packed_of(q, z.astype(np.uint8), s, zeros).to(DEV)
    lay = binding.mpq_g4_layout(32, d, group, zeros)
    values = ref.g4_values(q, z, s, d)
    got = binding.mpq_g4_dequantize(packed, lay)
    assert np.array_equal(got.cpu().numpy(), values.astype(np.float32))
    for T in (3, 40, 300):
        x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
        y = binding.mpq_g4_linear(x.to(DEV), packed, lay, dtype=torch.float32)
        w = torch.from_numpy(values).to(torch.float32).to(torch.bfloat16).double()     # (exact in fp32)
        tol = (d + 16) * 2.0 ** -23 * (x.double().abs() @ w.abs().T)
        assert bool(((y.cpu().double() - x.double() @ w.T).abs() <= tol).all())


def layer(T, C, d, group, zeros, dtype, out, bias, seed, pad=0, shift=0):
    """(call, exact outputs, bounds) of a layer; rows of x and y `pad` elements apart from `shift` on."""
    x = inputs(T, d, seed, dtype)
    w = 0.05 * inputs(C, d, seed + 1, shift=0.5 if zeros else 0.0)
    lay = binding.mpq_g4_layout(C, d, group, zeros)
    packed = binding.mpq_g4_quantize(w.to(DEV), lay)
    flat = torch.full((shift + T * (d + pad) + 8,), float("nan"), dtype=TYPES[dtype], device=DEV)
    rows = flat[shift:shift + T * (d + pad)].view(T, d + pad)[:, :d]
    rows.copy_(x)
    b = torch.randn(C, generator=torch.Generator().manual_seed(seed)).to(DEV) if bias else None
    xv, wv = x.to(DEV).double(), binding.mpq_g4_dequantize(packed, lay, dtype=TYPES[dtype]).double()
    want = xv @ wv.T
    tol = (d + 16) * 2.0 ** -23 * (xv.abs() @ wv.abs().T)
    if bias:
        want = want + b.double()
        tol = tol + 2.0 ** -23 * (want.abs() + b.double().abs())
    tol = tol + UNIT[out] * (want.abs() + tol) + (2.0 ** -25 if out == "fp16" else 0.0)
    call = lambda **k: binding.mpq_g4_linear(rows, packed, lay, bias=b, **(k or dict(dtype=TYPES[out])))
    return call, want, tol


def within(y, want, tol):
    """Every output within its bound; past fp16's largest number, the infinity it rounds to."""
    y, most = y.double(), torch.finfo(y.dtype).max
    over = want.abs() - tol > most * (1 + 2.0 ** -11)
    near = ((y - want).abs() <= tol) | (y.isinf() & (want.abs() + tol > most) & (y * want > 0))
    return bool((near & (~over | y.isinf())).all())


@pytest.mark.parametrize("T,C,d", [
    (1, 1, 1), (1, 16, 128), (1, 300, 4096), (2, 17, 129), (7, 129, 257), (8, 500, 640), (9, 33, 1000),
    (16, 4096, 512), (17, 640, 1000), (33, 500, 64), (31, 127, 2176), (63, 256, 384), (65, 130, 512),
    (75, 520, 4096), (128, 128, 256), (129, 384, 640), (200, 64, 2560), (256, 256, 1024), (257, 129, 136),
    (700, 300, 776), (1030, 1030, 304), (3, 20000, 128), (513, 3001, 1000), (2100, 2050, 512), (5000, 300, 128),
    (256, 4096, 4096), (208, 200, 9000), (250, 2000, 11008), (30, 600, 11000), (600, 700, 8200),
    (300, 100, 1), (150, 20, 7), (200, 1, 4096), (129, 17, 65), (1000, 129, 33), (4000, 40, 200)])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
def test_linear(gpu, T, C, d, group, zeros):
    dtype, out = ("bf16", "fp16")[(T + C) % 2], list(TYPES)[(T + C + group // 32) % 3]
    call, want, tol = layer(T, C, d, group, zeros, dtype, out, (T + d) % 2 == 0, T + C + d)
    y = call()
    assert y.shape == (T, C) and y.dtype == TYPES[out]
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())
    assert binding.mpq_device_status() == 0


@pytest.mark.parametrize("group,zeros", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [4, 24, 60, 300])
def test_linear_kinds(gpu, T, dtype, group, zeros):
    call, want, tol = layer(T, 200, 1152, group, zeros, dtype, "fp32", True, T + group)
    y = call()
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())


@pytest.mark.parametrize("T,C,d,pad,shift", [
    (1, 40, 131, 0, 1), (1, 40, 136, 0, 4), (5, 100, 333, 0, 0), (5, 100, 320, 3, 0), (12, 77, 320, 8, 1),
    (40, 77, 333, 2, 0), (100, 200, 1027, 0, 0), (90, 200, 1024, 8, 0), (300, 260, 333, 5, 3), (1100, 300, 258, 0, 0)])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, False)])
def test_linear_odd_rows(gpu, T, C, d, pad, shift, group, zeros):
    """Rows of x off the 16-byte boundary, of odd lengths and further apart; what lies between is not read
    into a sum (it is NaN)."""
    call, want, tol = layer(T, C, d, group, zeros, "bf16", "bf16", False, T + C, pad, shift)
    y = call()
    assert within(y, want, tol), float(((y.double() - want).abs() / tol).max())


@pytest.mark.parametrize("T,C,d", [(1, 256, 4096), (20, 300, 8000), (60, 129, 1000), (300, 203, 600), (1600, 1301, 304)])
def test_linear_repeats_bits_and_leaves_the_rest(gpu, T, C, d):
    """Equal bits from call to call; rows of the output further apart: nothing is written between them or past
    the last."""
    call, _, _ = layer(T, C, d, 128, False, "bf16", "bf16", False, 11)
    y = call()
    for pad in (0, 3, 5):
        buf = torch.full((T + 1, C + pad), 3.0, dtype=torch.bfloat16, device=DEV)
        for _ in range(2):
            call(Y=buf[:T, :C])
            assert torch.equal(buf[:T, :C], y)
        assert bool((buf[:, C:] == 3.0).all()) and bool((buf[T] == 3.0).all())


@pytest.mark.parametrize("T", [3, 30, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_weights_of_every_size(gpu, T, dtype):
    """Scales over the range of bf16, in fp16 too those whose values are subnormal, vanish or overflow: the values
    that the matrix stands for in x's type, bit for bit (x is one row of the identity at a time)."""
    d = 64
    s = np.exp2(np.arange(-140, 126, dtype=np.float64)).astype(np.float32)
    s = ref.bf16(np.concatenate([s, s * 1.5078125, -s * 1.9921875]))[:, None].repeat(d // 32, 1)
    q = np.random.default_rng(1).integers(0, 16, (len(s), d)).astype(np.uint8)
    z = np.random.default_rng(2).integers(0, 16, s.shape).astype(np.uint8)
    pad = lambda a, n: np.concatenate([a, np.zeros((len(a), n), a.dtype)], 1)
    packed = packed_of(pad(q, 64), pad(z, 2), pad(s, 2), True).to(DEV)
    lay = binding.mpq_g4_layout(len(s), d, 32, True)
    want = binding.mpq_g4_dequantize(packed, lay, dtype=TYPES[dtype])
    x = torch.zeros(T, d, dtype=TYPES[dtype], device=DEV)
    rows = torch.arange(T, device=DEV) % d
    x[torch.arange(T, device=DEV), rows] = 1
    finite = torch.isfinite(want).all(1)                            # (0 times infinity is NaN)
    y = binding.mpq_g4_linear(x, packed, lay, dtype=torch.float32)
    small = want.abs() < 2.0 ** -126                                # (fp32 sums may drop their subnormals)
    got = y[:, finite].T
    assert torch.equal(torch.where(small[finite][:, rows], 0.0, got),
                       torch.where(small, torch.zeros_like(want), want)[finite][:, rows].float())


@pytest.mark.parametrize("T", [5, 24, 130, 1500])
def test_linear_nan_and_infinity(gpu, T):
    """A NaN of the inputs makes its row NaN, a NaN group of the weights its column, nothing else; an infinity's
    row is infinite or NaN."""
    C, d = 140, 512
    x, w = inputs(T, d, 1, "bf16"), inputs(C, d, 2)
    x[3, 400] = float("nan")
    w[137, 5] = float("nan")
    lay = binding.mpq_g4_layout(C, d, 64, False)
    packed = binding.mpq_g4_quantize(w.to(DEV), lay)
    y = binding.mpq_g4_linear(x.to(DEV), packed, lay, dtype=torch.float32)
    bad = torch.zeros(T, C, dtype=torch.bool, device=DEV)
    bad[3], bad[:, 137] = True, True
    assert torch.equal(torch.isnan(y), bad)
    x[3, 400] = float("inf")
    y = binding.mpq_g4_linear(x.to(DEV), packed, lay, dtype=torch.float32)
    assert not bool(torch.isfinite(y[3]).any()) and torch.equal(torch.isfinite(y), ~bad)


def test_empty_and_streams(gpu):
    lay0, lay = binding.mpq_g4_layout(0, 64, 32), binding.mpq_g4_layout(40, 64, 32)
    p0 = binding.mpq_g4_quantize(torch.empty(0, 64, device=DEV), lay0)
    assert p0.numel() == 0 and binding.mpq_g4_dequantize(p0, lay0).shape == (0, 64)
    w, x = inputs(40, 64, 3).to(DEV), inputs(30, 64, 4, "bf16").to(DEV)
    p = binding.mpq_g4_quantize(w, lay)
    assert binding.mpq_g4_linear(x[:0], p, lay).shape == (0, 40)
    assert binding.mpq_g4_linear(x, p0, lay0).shape == (30, 0)
    want = binding.mpq_g4_linear(x, p, lay)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = binding.mpq_g4_linear(x, binding.mpq_g4_quantize(w, lay, stream=side), lay, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [1, 30, 400])
def test_chain_of_dependent_calls_and_its_graph(gpu, T):
    """Calls that follow one another on a stream, each reading what the one before has written, singly and
    as a graph's replay."""
    d = 776
    lay = binding.mpq_g4_layout(d, d, 64, True)
    w = binding.mpq_g4_quantize((0.04 * inputs(d, d, 10)).to(DEV), lay)
    x = inputs(T, d, 9, "bf16").to(DEV)
    want = x
    for _ in range(4):
        want = binding.mpq_g4_linear(want, w, lay)
        torch.cuda.synchronize()

    def chain():
        y = x
        for _ in range(4):
            y = binding.mpq_g4_linear(y, w, lay)
        return y
    for _ in range(5):
        assert torch.equal(chain(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = chain()
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)


def test_refusals(gpu):
    x = torch.zeros(4, 64, device=DEV)
    lay = binding.mpq_g4_layout(4, 64, 32)
    p = binding.mpq_g4_quantize(x, lay)
    b = x.to(torch.bfloat16)
    for wrong in (x.int(), ):
        with pytest.raises(TypeError):
            binding.mpq_g4_quantize(wrong, lay)
    for wrong in (x.cpu(), x[:, :32], x[:2], torch.zeros(64, 4, device=DEV).T):
        with pytest.raises(ValueError):
            binding.mpq_g4_quantize(wrong, lay)
    with pytest.raises(ValueError):
        binding.mpq_g4_dequantize(p[:100], lay)
    with pytest.raises(ValueError):
        binding.mpq_g4_linear(b, p[:100], lay)
    with pytest.raises(binding.MPQError):
        binding.mpq_g4_linear(x, p, lay)                               # fp32 inputs
    for wrong in (b[:, :32], b[0], torch.zeros(64, 4, device=DEV, dtype=torch.bfloat16).T):
        with pytest.raises(ValueError):
            binding.mpq_g4_linear(wrong, p, lay)
    with pytest.raises(TypeError):
        binding.mpq_g4_linear(b, p, lay, bias=torch.zeros(4, device=DEV, dtype=torch.float16))
    with pytest.raises(ValueError):
        binding.mpq_g4_linear(b, p, lay, bias=torch.zeros(5, device=DEV))
    with pytest.raises(ValueError):
        binding.mpq_g4_linear(b, p, lay, Y=torch.zeros(4, 5, device=DEV))
    with pytest.raises(TypeError):
        binding.mpq_g4_linear(b, p, lay, Y=torch.zeros(4, 4, device=DEV, dtype=torch.int32))
    with pytest.raises(binding.MPQError):
        binding.mpq_g4_layout(4, 64, 48)


@pytest.mark.parametrize("T,C,d", [(140, 300, 512), (140, 300, 4096), (200, 500, 300), (700, 4000, 300)])
def test_linear_withheld_copies_time_out(gpu, T, C, d):
    """With the test hook on, the kernel's waits run out with nothing in flight: the status says so, and the
    same call is right again after (K whole, K split over a cluster, CTA pairs)."""
    call, _, _ = layer(T, C, d, 64, False, "bf16", "bf16", False, 3)
    good = call()
    assert binding.mpq_device_status() == 0
    try:
        binding.mpq_set_wait_limit(1 << 18)
        binding.mpq_test_withhold_copies(True)
        call()
        flags = binding.mpq_device_status()
    finally:
        binding.mpq_test_withhold_copies(False)
        binding.mpq_set_wait_limit(0)
    assert flags == binding.MPQ_TIMEOUT_G4
    assert torch.equal(call(), good)
    assert binding.mpq_device_status() == 0
