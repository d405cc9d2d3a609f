"""Norms of queries and keys with the position rotation on the GPU, against the formulas in 64 bits.

An element's bound, in units 2^-24 of the magnitudes that go into it (|x| of a plain element, |a| + |b| of a rotated
one): the norm's sum of squares is off by 16 additions of a thread and 5 across threads, the mean by two operations
more (all halved by the root), the root and two products by 3: 15; cosine and sine by 4 (2^-22), the
rotation's products and sum by 2.  The output's rounding adds 2^-24, 2^-11 or 2^-8 of |y| (fp32, fp16, bf16;
fp16 also 2^-25 absolutely)."""
import numpy as np
import pytest
import torch

import _decode_step as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def heads_of(T, heads, dim, seed, dtype):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, heads, dim)) * np.exp(rng.uniform(-2, 2, (T, heads, 1)))
    return torch.from_numpy(x).to(TYPES[dtype])


def frequencies(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / max(rot, 1))


def check(y, x, positions, freq, norm, weight, eps, neighbours, dtype):
    want, mag = ref.rotate(x.double().numpy(), positions, freq, norm,
                           None if weight is None else weight.double().numpy(), eps, neighbours)
    tol = 21 * 2.0 ** -24 * mag + UNIT[dtype] * np.abs(want) * (1 + 2.0 ** -19) + \
        (2.0 ** -25 if dtype == "fp16" else 0.0)
    off = np.abs(y.cpu().double().numpy() - want)
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("T,q_heads,heads,dim,rot", [
    (1, 1, 1, 2, 2), (3, 4, 2, 64, 64), (48, 32, 8, 128, 128), (5, 8, 8, 128, 64), (7, 3, 1, 80, 80),
    (9, 5, 5, 96, 48), (2, 16, 1, 256, 256), (33, 6, 2, 80, 40), (4, 2, 2, 512, 512), (6, 3, 3, 50, 26),
    (200, 1, 1, 128, 128), (4, 2, 1, 64, 0), (2, 70, 70, 128, 128), (1, 1, 1, 512, 2), (1000, 2, 1, 16, 16),
    (3, 40, 4, 512, 510)])
def test_rotate(gpu, T, q_heads, heads, dim, rot, norm, neighbours):
    dtype = list(TYPES)[(T + dim + norm) % 3]
    q, k = heads_of(T, q_heads, dim, T + dim, dtype), heads_of(T, heads, dim, T + dim + 1, dtype)
    freq, rng = frequencies(rot), np.random.default_rng(T)
    pos = rng.integers(0, 1 << 20, T)
    pos[0] = 0
    w = lambda i: torch.from_numpy(rng.standard_normal(dim)).float() if norm and (T + i) % 3 else None
    wq, wk = w(0), w(1)
    dev = lambda t: None if t is None else t.to(DEV)
    turns = binding.mpq_rotation(freq, DEV)
    yq, yk = binding.mpq_rotate(q.to(DEV), k.to(DEV), torch.from_numpy(pos).int().to(DEV), turns, norm=norm,
                                q_weight=dev(wq), k_weight=dev(wk), eps=1e-6, neighbours=neighbours)
    check(yq, q, pos, freq, norm, wq, 1e-6, neighbours, dtype)
    check(yk, k, pos, freq, norm, wk, 1e-6, neighbours, dtype)


@pytest.mark.parametrize("shift", [0, 5, -3, 2 ** 31 - 1, -2 ** 31])
def test_far_and_negative_positions(gpu, shift):
    """Positions of the whole range with a shift: exact turns, so the far ones are as good as the near."""
    T, dim = 11, 64
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, -123456789, 2 ** 24 + 1, 7, 65537, 99], np.int64)
    x, freq = heads_of(T, 2, dim, 1, "fp32"), frequencies(dim)
    turns = binding.mpq_rotation(freq, DEV)
    y, none = binding.mpq_rotate(x.to(DEV), None, torch.from_numpy(pos).int().to(DEV), turns, shift=shift)
    assert none is None
    # the angle from whole numbers: (position + shift) turns, its top 62 bits
    whole = [int(t) for t in turns.cpu().numpy().astype(np.uint64)]
    angle = np.array([[((int(p) + shift) * t % 2 ** 64 >> 2) / 2.0 ** 62 * 2 * np.pi for t in whole] for p in pos])
    a, b = x.double().numpy()[..., :32], x.double().numpy()[..., 32:]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    want = np.concatenate([a * c - b * s, b * c + a * s], 2)
    mag = np.concatenate([np.abs(a) + np.abs(b)] * 2, 2)
    assert (np.abs(y.cpu().double().numpy() - want) <= 7 * 2.0 ** -24 * mag).all()


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,rot", [(128, 128), (80, 40), (64, 12)])
def test_parts_of_a_projection_and_in_place(gpu, dtype, dim, rot, neighbours):
    """Queries and keys as views of one buffer, rows off the 16-byte boundary too, outputs there or elsewhere:
    equal bits, the values untouched."""
    T, hq, h = 21, 4, 2
    rows = heads_of(T, hq + 2 * h, dim, 3, dtype).to(DEV)
    pos = torch.arange(T, device=DEV, dtype=torch.int32) * 1000
    turns = binding.mpq_rotation(frequencies(rot), DEV)
    w = torch.rand(dim, device=DEV) + 0.5
    go = lambda q, k, **o: binding.mpq_rotate(q, k, pos, turns, norm=True, q_weight=w, k_weight=w,
                                              neighbours=neighbours, **o)
    q, k, v = rows.split((hq, h, h), 1)
    wq, wk = go(q.contiguous(), k.contiguous())
    for shift in (0, 1):
        flat = torch.full((rows.numel() + shift,), 9.0, dtype=rows.dtype, device=DEV)
        view = flat[shift:].view(rows.shape)
        view.copy_(rows)
        q, k, v = view.split((hq, h, h), 1)
        yq, yk = go(q, k)
        assert torch.equal(yq, wq) and torch.equal(yk, wk) and torch.equal(view, rows)
        r = go(q, k, Yq=q, Yk=k)
        assert r[0] is q and r[1] is k
        assert torch.equal(q, wq) and torch.equal(k, wk) and torch.equal(v, rows[:, hq + h:])
        by_head = torch.empty(hq, T, dim, dtype=rows.dtype, device=DEV).transpose(0, 1)
        view.copy_(rows)
        go(q, k, Yq=by_head)
        assert torch.equal(by_head, wq)


def test_norm_of_large_small_and_odd_values(gpu):
    """Squares past fp32's range, zeros (whose norm is eps alone), a NaN and an infinity, each in its row alone."""
    x = torch.randn(8, 1, 64, generator=torch.Generator().manual_seed(1))
    for i, f in enumerate((1e30, 3e37, 1e-20, 0.0, 1.0, 1.0, 2.0 ** 66, 1.0)):
        x[i] *= f
    x[4, 0, 5], x[5, 0, 9] = float("nan"), float("inf")
    pos = torch.arange(8, device=DEV, dtype=torch.int32)
    freq = frequencies(32)
    y, _ = binding.mpq_rotate(x.to(DEV), None, pos, binding.mpq_rotation(freq, DEV), norm=True, eps=1e-6)
    good = [0, 1, 2, 3, 6, 7]
    check(y[good], x[good], np.array(good), freq, True, None, 1e-6, False, "fp32")
    assert bool(y[4].isnan().all())
    # x / sqrt(mean) is NaN at the infinity (and what is turned with it), zero elsewhere
    bad = torch.zeros(64, dtype=torch.bool)
    bad[[9, 25]] = True
    assert torch.equal(y[5, 0].cpu().isnan(), bad) and bool((y[5, 0].cpu()[~bad] == 0).all())


def test_one_side_none_and_empty(gpu):
    x = heads_of(4, 2, 64, 1, "bf16").to(DEV)
    pos = torch.arange(4, device=DEV, dtype=torch.int32)
    turns = binding.mpq_rotation(frequencies(64), DEV)
    q, k = binding.mpq_rotate(x, x, pos, turns)
    alone, none = binding.mpq_rotate(x, None, pos, turns)
    assert none is None and torch.equal(alone, q) and torch.equal(k, q)
    assert binding.mpq_rotate(x[:0], x[:0], pos[:0], turns)[0].shape == (0, 2, 64)
    assert binding.mpq_rotate(x[:, :0], x, pos, turns)[0].shape == (4, 0, 64)
    still, _ = binding.mpq_rotate(x, None, pos, turns[:0])
    assert torch.equal(still, x)


def test_stream_and_graph(gpu):
    x = heads_of(40, 8, 128, 1, "bf16").to(DEV)
    pos = torch.arange(40, device=DEV, dtype=torch.int32)
    turns = binding.mpq_rotation(frequencies(128), DEV)
    want, _ = binding.mpq_rotate(x, None, pos, turns, norm=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, _ = binding.mpq_rotate(x, None, pos, turns, norm=True, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = binding.mpq_rotate(x, None, pos, turns, norm=True)
    pos += 3
    graph.replay()
    assert torch.equal(got, binding.mpq_rotate(x, None, pos - 3, turns, norm=True, shift=3)[0])


def test_refusals(gpu):
    x = heads_of(4, 2, 64, 1, "bf16").to(DEV)
    pos = torch.arange(4, device=DEV, dtype=torch.int32)
    turns = binding.mpq_rotation(frequencies(64), DEV)
    go = binding.mpq_rotate
    for bad in ((x, x[:3], pos, turns), (x, x[..., :32], pos, turns), (x, x.float(), pos, turns),
                (x, x, pos[:3], turns), (x, x, pos, turns[None]), (x[0], None, pos, turns),
                (x.transpose(1, 2), None, pos, turns), (x.cpu(), None, pos, turns)):
        with pytest.raises(ValueError):
            go(*bad)
    for bad in ((x, x, pos.long(), turns), (x, x, pos, turns.float()), (x.int(), None, pos, turns), (None, x, pos, turns)):
        with pytest.raises(TypeError):
            go(*bad)
    with pytest.raises(binding.MPQError):
        go(x, x, pos, torch.cat([turns, turns]))                       # rot > dim
    with pytest.raises(binding.MPQError):
        go(x, x, pos, turns, q_weight=torch.ones(64, device=DEV))      # weights without a norm
    with pytest.raises(binding.MPQError):
        go(x, x, pos, turns, norm=True, eps=0.0)
    with pytest.raises(ValueError):
        go(x, x, pos, turns, norm=True, q_weight=torch.ones(32, device=DEV))
    with pytest.raises(ValueError):
        go(x, None, pos, turns, Yk=x)
    with pytest.raises(TypeError):
        go(x, None, pos, turns, Yq=x.float())
    with pytest.raises(binding.MPQError):
        go(x, None, pos, turns, Yq=torch.empty(1, 2, 64, device=DEV, dtype=x.dtype).expand(4, 2, 64))
