"""The few-bit key-value cache on the GPU: what is written and read back, bit for bit against the
definition's fp32 operations, and the attention of one new token against 64-bit sums over the same
cached values.

The attention's bound, per output element, with A = sum p |v| / sum p in 64 bits: the weights are
rounded to fp16 (2^-11 A); a score is off by at most (dim + 2) 2^-23 of sum |q k| scale, and each
exponential, logarithm and scale factor by a few fp32 units, 2^-20 in all, which move a weight and the
sum by that relative amount each; weights below 2^-14 of fp16's range are off by 2^-25, at least 2^-31
of the largest weighted value for each attended token; the output's own rounding adds half a unit."""
import math

import numpy as np
import pytest
import torch

import _serving as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def stored(codes, scales, slots, lay):
    """(codes q, scales) [T][2][heads] of slots, from the cache's storage."""
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    p, at = np.divmod(np.asarray(slots), lay.page)
    rows = c[p, :, :, at]
    if lay.bits == 4:
        rows = np.stack([rows & 15, rows >> 4], -1).reshape(rows.shape[:-1] + (lay.dim,))
    return rows.astype(np.int32) - (1 << (lay.bits - 1)), s[p, :, :, at]


def tokens(T, heads, dim, seed, dtype):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((2, T, heads, dim)) * np.exp(rng.uniform(-2, 2, (2, T, heads, 1)))
    return torch.from_numpy(x).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,heads,dim,bits,page", [
    (1, 1, 64, 8, 16), (7, 3, 128, 8, 16), (33, 2, 256, 8, 48), (5, 8, 64, 4, 32),
    (130, 1, 128, 4, 16), (9, 5, 256, 4, 1024)])
def test_write_and_read_back(gpu, T, heads, dim, bits, page, dtype):
    lay = binding.mpq_cache_layout(T // page + 2, page, heads, dim, bits)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    codes.fill_(0xA5)
    scales.fill_(-3.0)
    x = tokens(T, heads, dim, T + dim, dtype)
    perm = np.random.default_rng(1).permutation(lay.pages * page)
    slots = torch.from_numpy(perm[:T]).to(DEV)
    binding.mpq_cache_write(x[0].to(DEV), x[1].to(DEV), slots, lay, codes, scales)
    q, s = stored(codes, scales, perm[:T], lay)
    q_ref, s_ref = ref.cache_rows(x.float().numpy(), bits)
    assert np.array_equal(q, q_ref.transpose(1, 0, 2, 3)) and \
        np.array_equal(s, s_ref.transpose(1, 0, 2))
    rest = perm[T:]                                  # nothing else was touched
    p, at = np.divmod(rest, page)
    assert (codes.cpu().numpy()[p, :, :, at] == 0xA5).all()
    assert (scales.cpu().numpy()[p, :, :, at] == -3.0).all()
    want = torch.from_numpy(q_ref.astype(np.float32) * s_ref[..., None])
    for t in TYPES.values():
        K, V = binding.mpq_cache_read(slots, lay, codes, scales, dtype=t)
        assert torch.equal(K.cpu(), want[0].to(t)) and torch.equal(V.cpu(), want[1].to(t))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shift", [0, 1])
def test_write_strided(gpu, dtype, shift):
    """Keys and values as parts of one projection's output, also off the 16-byte boundary."""
    T, heads, dim = 20, 2, 64
    lay = binding.mpq_cache_layout(3, 16, heads, dim, 8)
    x = tokens(T, heads, dim, 3, dtype).to(DEV)
    wide = torch.full((T * 5 * heads * dim + 8,), float("nan"), dtype=TYPES[dtype], device=DEV)
    rows = wide[shift:shift + T * 5 * heads * dim].view(T, 5 * heads, dim)
    K, V = rows[:, heads:2 * heads], rows[:, 3 * heads:4 * heads]
    K.copy_(x[0])
    V.copy_(x[1])
    slots = torch.arange(T, device=DEV) + 9
    a, b = binding.mpq_cache_empty(lay, DEV), binding.mpq_cache_empty(lay, DEV)
    binding.mpq_cache_write(K, V, slots, lay, *a)
    binding.mpq_cache_write(x[0], x[1], slots, lay, *b)
    for u, v in zip(binding.mpq_cache_read(slots, lay, *a), binding.mpq_cache_read(slots, lay, *b)):
        assert torch.equal(u, v)


@pytest.mark.parametrize("bits", [8, 4])
def test_slots_outside_and_special_rows(gpu, bits):
    """Slots outside the cache are skipped and read as zeros; rows of zeros, subnormals, infinities
    and NaN; halfway cases round to even."""
    dim, qmax = 64, 2 ** (bits - 1) - 1
    lay = binding.mpq_cache_layout(2, 16, 1, dim, bits)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    codes.zero_()
    scales.zero_()
    x = np.zeros((9, dim), np.float32)
    x[1] = np.linspace(-1, 1, dim)
    x[2, 5] = 2.0 ** -149                           # the scale underflows
    x[3] = np.linspace(-1, 1, dim) * 2.0 ** -140    # a subnormal scale
    x[4], x[4, 7] = 1.0, np.inf
    x[5], x[5, 8] = 1.0, np.nan
    x[6] = (np.arange(dim) % (2 * qmax) - qmax + 0.5)
    x[6, 0] = qmax                                   # scale 1: every other element a tie
    x[7] = 3e38
    x[8] = 5.0
    slot = np.array([3, 31, 0, 7, 8, 9, 10, 11, 32])
    kv = torch.from_numpy(x).to(DEV).view(9, 1, dim)
    binding.mpq_cache_write(kv, -kv, torch.from_numpy(slot).to(DEV), lay, codes, scales)
    before = codes.clone()
    binding.mpq_cache_write(kv, kv, torch.tensor([-1, 32, -2 ** 62, 2 ** 62, 33, 34, 35, 36, 37],
                                                 device=DEV), lay, codes, scales)
    assert torch.equal(before, codes)
    q, s = stored(codes, scales, slot[:8], lay)
    q_ref, s_ref = ref.cache_rows(x[:8], bits)
    assert np.array_equal(q[:, 0, 0], q_ref) and np.array_equal(q[:, 1, 0], -q_ref)
    assert np.array_equal(s[:, 0, 0], s_ref, equal_nan=True)
    K, V = binding.mpq_cache_read(torch.tensor([-1, 3, 32, 31], device=DEV), lay, codes, scales,
                                  dtype=torch.float32)
    assert bool((K[0] == 0).all()) and bool((V[2] == 0).all())
    assert np.array_equal(K[3, 0].cpu().numpy(), q_ref[1].astype(np.float32) * s_ref[1])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_write_quotients_near_halves(gpu, bits, dtype):
    """Elements a few units around every half of the scale, and simple fractions of the largest: the
    codes are those of the correctly rounded fp32 quotients."""
    dim, T, qmax = 256, 600, 2 ** (bits - 1) - 1
    rng = np.random.default_rng(bits)
    top = np.exp(rng.uniform(-9, 9, (T, 1))).astype(np.float32)
    if dtype == "fp16":
        top = top.astype(np.float16).astype(np.float32)
    s = top * (np.float32(1) / np.float32(qmax))
    half = rng.integers(0, qmax, (T, dim)) + 0.5
    x = (s * half).astype(np.float32)
    x = (x.view(np.int32) + rng.integers(-3, 4, (T, dim))).astype(np.int32).view(np.float32)
    x[:, ::5] = (top * rng.integers(0, 2 * qmax, (T, dim)) / (2 * qmax)).astype(np.float32)[:, ::5]
    x = np.minimum(x, top) * rng.choice([-1, 1], (T, dim)).astype(np.float32)
    x[:, 0] = top[:, 0]
    x = torch.from_numpy(x).to(TYPES[dtype])
    lay = binding.mpq_cache_layout(-(-T // 16), 16, 1, dim, bits)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    kv = x.to(DEV).view(T, 1, dim)
    binding.mpq_cache_write(kv, -kv, torch.arange(T, device=DEV), lay, codes, scales)
    q, sc = stored(codes, scales, np.arange(T), lay)
    q_ref, s_ref = ref.cache_rows(x.float().numpy(), bits)
    assert np.array_equal(sc[:, 0, 0], s_ref) and np.array_equal(sc[:, 1, 0], s_ref)
    assert np.array_equal(q[:, 0, 0], q_ref) and np.array_equal(q[:, 1, 0], -q_ref)


class Scene:
    """A cache filled at random (NaN scales wherever no sequence looks), its tables, and the queries."""

    def __init__(self, lens, heads, group, dim, bits, page, dtype, seed, spare=2, cols=None,
                 loud=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.heads, self.group, self.dim = lens, heads, group, dim
        self.page, self.dtype = page, dtype
        need = [-(-n // page) for n in lens]
        self.lay = binding.mpq_cache_layout(sum(need) + spare, page, heads, dim, bits)
        order = rng.permutation(self.lay.pages)
        self.table = np.full((len(lens), cols or max(1, max(need))), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        qmax = 2 ** (bits - 1) - 1
        self.codes = rng.integers(-qmax, qmax + 1, (self.lay.pages, 2, heads, page, dim))
        self.scales = np.exp(rng.uniform(-6, -3, (self.lay.pages, 2, heads, page))).astype(np.float32)
        for b, n in enumerate(lens):
            if n % page:
                self.scales[self.table[b, n // page], :, :, n % page:] = np.nan
        used = np.zeros(self.lay.pages, bool)
        used[self.table[self.table >= 0]] = True
        self.scales[~used] = np.nan
        q = loud * rng.standard_normal((len(lens), heads * group, dim))
        self.q = torch.from_numpy(q).to(TYPES[dtype])
        raw = self.codes + (1 << (bits - 1))
        if bits == 4:
            raw = raw[..., 0::2] | (raw[..., 1::2] << 4)
        self.d_codes = torch.from_numpy(raw.astype(np.uint8)).to(DEV)

    def run(self, window=0, scale=None, q=None, lens=None, lse=True, workspace=None):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        B = len(self.lens)
        out = torch.full((B, self.heads * self.group), 9.0, device=DEV) if lse else None
        o = binding.mpq_cache_attention(
            self.q.to(DEV) if q is None else q, t(self.table),
            t(np.array(self.lens if lens is None else lens, np.int32)), self.lay, self.d_codes,
            t(self.scales), scale=scale, window=window, lse=out, workspace=workspace)
        return o, out

    def check(self, o, lse, window=0, scale=None, heads=None):
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        o, lse = o.cpu().double().numpy(), lse.cpu().double().numpy()
        q = self.q.double().numpy()
        for b, n in enumerate(self.lens):
            t = np.arange(n)
            page = self.table[b, t // self.page] if n else np.zeros(0, np.int32)
            seen = (page >= 0) & (page < self.lay.pages)
            if window:
                seen &= t >= n - window
            page = np.where(seen, page, 0)
            for h in heads or range(self.heads):
                kv = [self.codes[page, i, h, t % self.page].astype(np.float64) *
                      self.scales[page, i, h, t % self.page].astype(np.float64)[:, None]
                      for i in (0, 1)]
                for j in range(h * self.group, (h + 1) * self.group):
                    want, l, A, unit, reach = ref.attention(q[b, j], kv[0], kv[1], seen, scale)
                    drift = (self.dim + 2) * 2.0 ** -23 * reach + 2.0 ** -20
                    tol = A * (2.0 ** -11 + 4 * drift) + int(seen.sum()) * 2.0 ** -31 * unit
                    tol = tol + UNIT[self.dtype] * (np.abs(want) + tol) + 2.0 ** -25
                    assert (np.abs(o[b, j] - want) <= tol).all(), \
                        (b, h, j, float((np.abs(o[b, j] - want) / tol).max()))
                    if np.isinf(l):
                        assert lse[b, j] == -np.inf and not o[b, j].any()
                    else:
                        assert abs(lse[b, j] - l) <= drift + 2.0 ** -22 * abs(l)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("group", [1, 3, 8, 9, 16, 20])
def test_attention_shapes(gpu, dim, bits, group):
    s = Scene([65, 0, 1, 200, 16], 2, group, dim, bits, 16, "bf16" if group % 2 else "fp16",
              dim + bits + group, loud=2.0)
    o, lse = s.run()
    s.check(o, lse)


@pytest.mark.parametrize("page", [16, 48, 64, 1024])
@pytest.mark.parametrize("lens", [[1], [17], [63, 64, 65], [1023, 1024, 1025], [5, 3000, 0, 0, 129]])
def test_attention_lengths_and_pages(gpu, page, lens):
    s = Scene(lens, 1, 4, 128, 8, page, "bf16", page + sum(lens), loud=3.0)
    o, lse = s.run()
    s.check(o, lse)


@pytest.mark.parametrize("heads,lens", [(1, [9000]), (3, [4097, 20]), (2, [0, 6000, 1, 6000])])
@pytest.mark.parametrize("bits,dim", [(8, 128), (4, 64)])
def test_attention_split_rows_join(gpu, heads, lens, bits, dim):
    """Rows long enough that many CTAs share one; the same bits from call to call, with the caller's
    workspace (used again) and without."""
    s = Scene(lens, heads, 5, dim, bits, 32, "fp16", 17 + heads, loud=2.0)
    ws = torch.zeros(binding.MPQ_CACHE_WORKSPACE, dtype=torch.uint8, device=DEV)
    o, lse = s.run(workspace=ws)
    s.check(o, lse)
    for w in (ws, ws, None):
        o2, lse2 = s.run(workspace=w)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("window", [1, 16, 63, 64, 65, 130, 5000])
def test_attention_window(gpu, window):
    s = Scene([1, 64, 300, 0, 1000], 2, 4, 64, 8, 16, "bf16", window)
    o, lse = s.run(window=window)
    s.check(o, lse, window=window)


def test_attention_many_sequences(gpu):
    lens = list(np.random.default_rng(4).integers(0, 90, 300))
    s = Scene([int(n) for n in lens], 1, 2, 64, 8, 16, "bf16", 8)
    o, lse = s.run()
    s.check(o, lse)


def test_attention_missing_pages(gpu):
    """Table entries that name no page hold nothing to attend to; a sequence of such pages only is
    an empty row; lengths beyond the table or below zero are cut to it."""
    s = Scene([100, 64, 200, 48], 2, 3, 128, 8, 16, "bf16", 5)
    s.table[0, 2], s.table[0, 4] = -1, s.lay.pages
    s.table[1, :] = -7
    s.table[3, 0] = 2 ** 31 - 1
    o, lse = s.run()
    s.check(o, lse)
    cols = s.table.shape[1]
    s2 = Scene([cols * 16], 2, 3, 128, 8, 16, "bf16", 6)
    o, lse = s2.run(lens=[cols * 16 + 1000])
    s2.check(o, lse)
    o, lse = s2.run(lens=[-5])
    assert not o.any() and bool((lse == -math.inf).all())


def test_attention_scales_of_all_sizes(gpu):
    """Value scales from 2^-60 to 2^60 (a token's precision does not hang on its values' size), zero
    scales, and queries with elements far apart."""
    s = Scene([300, 70], 2, 4, 64, 8, 16, "bf16", 12, loud=4.0)
    rng = np.random.default_rng(3)
    live = np.isfinite(s.scales[:, 1])
    s.scales[:, 1] = np.where(live, np.exp2(rng.integers(-60, 60, live.shape)), np.nan)
    s.scales[s.table[0, 3], 1, 0, 4] = 0.0
    s.scales[s.table[0, 5], 0, 1, 2] = 0.0
    s.q[0, 0, :] *= 2.0 ** -20
    s.q[1, 1, 3] = 4000.0
    o, lse = s.run()
    s.check(o, lse)
    # one token among the attended whose value scale is 2^-40 of the others' takes all the weight
    s = Scene([200], 1, 2, 64, 8, 16, "bf16", 13)
    s.scales[s.table[0, 7], 1, 0, 0] = 2.0 ** -40
    s.scales[s.table[0, 7], 0, 0, 0] = 50.0
    o, lse = s.run()
    s.check(o, lse)


def test_attention_nan_reaches_its_heads_only(gpu):
    s = Scene([100, 90], 2, 2, 64, 8, 16, "bf16", 14)
    s.scales[s.table[0, 1], 1, 1, 3] = np.nan        # a value of sequence 0, key head 1
    s.scales[s.table[1, 2], 0, 0, 5] = np.nan        # a key of sequence 1, key head 0
    s.q[0, 0, 7] = float("nan")
    o, _ = s.run()
    bad = torch.isnan(o).all(-1).cpu()
    want = torch.zeros(2, 4, dtype=torch.bool)
    want[0, 2:], want[1, :2], want[0, 0] = True, True, True
    assert torch.equal(bad, want)
    assert torch.equal(torch.isnan(o).any(-1).cpu(), want)


@pytest.mark.parametrize("shift,stride", [(0, 7), (1, 0), (4, 4)])
def test_attention_strided_queries(gpu, shift, stride):
    s = Scene([40, 100], 2, 4, 128, 8, 16, "fp16", 15)
    B, H, D = s.q.shape
    buf = torch.full((shift + B * (H * D + stride),), float("nan"), dtype=s.q.dtype, device=DEV)
    q = buf[shift:].view(B, H * D + stride)[:, :H * D].view(B, H, D)
    q.copy_(s.q)
    o, lse = s.run(q=q)
    o2, lse2 = s.run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_attention_scale_and_streams(gpu):
    s = Scene([500], 1, 4, 64, 8, 16, "bf16", 16)
    for scale in (0.0, -0.3, 2.0):
        o, lse = s.run(scale=scale)
        s.check(o, lse, scale=scale)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2, lse2 = s.run(scale=2.0)
    side.synchronize()
    assert torch.equal(o, o2)


def test_attention_offsets_beyond_32_bits(gpu):
    """A cache of more than 2^32 bytes whose last pages are read, written and attended to."""
    heads, dim, page = 8, 256, 1024
    lay = binding.mpq_cache_layout(1100, page, heads, dim, 8)
    assert lay.codes_bytes > 2 ** 32
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    scales.fill_(math.nan)
    n = 70
    x = tokens(n, heads, dim, 5, "bf16")
    slots = torch.arange(n, device=DEV) + (lay.pages - 1) * page
    binding.mpq_cache_write(x[0].to(DEV), x[1].to(DEV), slots, lay, codes, scales)
    q_ref, s_ref = ref.cache_rows(x.float().numpy(), 8)
    want = q_ref * s_ref[..., None].astype(np.float64)
    K, V = binding.mpq_cache_read(slots, lay, codes, scales, dtype=torch.float32)
    assert np.array_equal(K.cpu().numpy(), want[0].astype(np.float32))
    q = torch.randn(1, heads, dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    o = binding.mpq_cache_attention(q.to(DEV), torch.tensor([[lay.pages - 1]], dtype=torch.int32,
                                                            device=DEV),
                                    torch.tensor([n], dtype=torch.int32, device=DEV), lay, codes,
                                    scales)
    for h in range(heads):
        r, _, A, unit, reach = ref.attention(q[0, h].double().numpy(), want[0][:, h], want[1][:, h],
                                             np.ones(n, bool), 1 / math.sqrt(dim))
        drift = (dim + 2) * 2.0 ** -23 * reach + 2.0 ** -20
        tol = A * (2.0 ** -11 + 4 * drift) + n * 2.0 ** -31 * unit
        tol = tol + 2.0 ** -8 * (np.abs(r) + tol)
        assert (np.abs(o[0, h].cpu().double().numpy() - r) <= tol).all()


def test_attention_withheld_copies_time_out(gpu):
    """With the test hook on, the kernel's waits run out with nothing in flight: outputs read NaN,
    the status says so, and the same call is right again after."""
    s = Scene([40, 700], 1, 4, 64, 8, 16, "bf16", 21)
    good, lse = s.run()
    assert binding.mpq_device_status() == 0
    try:
        binding.mpq_set_wait_limit(1 << 18)
        binding.mpq_test_withhold_copies(True)
        bad, _ = s.run()
        flags = binding.mpq_device_status()
    finally:
        binding.mpq_test_withhold_copies(False)
        binding.mpq_set_wait_limit(0)
    assert flags == binding.MPQ_TIMEOUT_ATTENTION
    assert bool(torch.isnan(bad).all())
    o, l = s.run()
    assert torch.equal(o, good) and torch.equal(l, lse) and binding.mpq_device_status() == 0


def test_refusals(gpu):
    lay = binding.mpq_cache_layout(4, 16, 2, 64, 8)
    codes, scales = binding.mpq_cache_empty(lay, DEV)
    K = torch.zeros(3, 2, 64, device=DEV)
    slots = torch.arange(3, device=DEV)
    with pytest.raises(ValueError):
        binding.mpq_cache_write(K, K[:, :1], slots, lay, codes, scales)
    with pytest.raises(ValueError):
        binding.mpq_cache_write(K, K.half(), slots, lay, codes, scales)
    with pytest.raises(TypeError):
        binding.mpq_cache_write(K, K, slots.int(), lay, codes, scales)
    with pytest.raises(ValueError):
        binding.mpq_cache_write(K, K, slots, lay, codes[:2], scales)
    with pytest.raises(TypeError):
        binding.mpq_cache_write(K.double(), K.double(), slots, lay, codes, scales)
    q = torch.zeros(2, 4, 64, device=DEV, dtype=torch.bfloat16)
    table = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    lens = torch.ones(2, dtype=torch.int32, device=DEV)
    att = lambda **k: binding.mpq_cache_attention(
        **dict(dict(Q=q, table=table, lens=lens, layout=lay, codes=codes, scales=scales), **k))
    with pytest.raises(binding.MPQError):
        att(Q=q.float())
    with pytest.raises(binding.MPQError):
        att(Q=q[:, :3])
    with pytest.raises(binding.MPQError):
        att(window=-1)
    with pytest.raises(binding.MPQError):
        att(scale=float("nan"))
    with pytest.raises(binding.MPQError):
        att(workspace=torch.zeros(1024, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        att(Q=q[:1])
    with pytest.raises(TypeError):
        att(lens=lens.long())
    for bad in ((-1, 16, 2, 64, 8), (4, 0, 2, 64, 8), (4, 24, 2, 64, 8), (4, 16, 0, 64, 8),
                (4, 16, 2, 96, 8), (4, 16, 2, 64, 5)):
        with pytest.raises(binding.MPQError):
            binding.mpq_cache_layout(*bad)
