"""A serving step made of the few-bit calls from the requests' lengths on -- room and slots for the new
tokens, the projection by 4-bit integer weights, norm and rotation, the cache's write, the attention, the projection
back -- for prompts, single tokens and requests that are cut back; eager and as one graph's replays."""
import math

import numpy as np
import pytest
import torch

import _decode_step as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, H, DIM, D, PAGE, PAGES, COLS = 8, 2, 64, 512, 16, 60, 12


class Layer:
    def __init__(self, group, zeros, dtype=torch.bfloat16):
        gen = torch.Generator(device=DEV).manual_seed(group + zeros)
        rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
        self.dtype, self.rand = dtype, rand
        w = lambda r, c: rand(r, c) / math.sqrt(c)
        self.in_layout = binding.mpq_g4_layout((HQ + 2 * H) * DIM, D, group, zeros)
        self.out_layout = binding.mpq_g4_layout(D, HQ * DIM, group, zeros)
        self.w_in = binding.mpq_g4_quantize(w((HQ + 2 * H) * DIM, D), self.in_layout)
        self.w_out = binding.mpq_g4_quantize(w(D, HQ * DIM), self.out_layout)
        self.cache = binding.mpq_cache_layout(PAGES, PAGE, H, DIM, 8)
        self.codes, self.scales = binding.mpq_cache_empty(self.cache, DEV)
        self.codes.zero_()
        self.scales.zero_()
        self.freq = 10000.0 ** (-np.arange(0, DIM, 2) / DIM)
        self.turns = binding.mpq_rotation(self.freq, DEV)
        self.q_weight, self.k_weight = rand(DIM).abs() + 0.5, rand(DIM).abs() + 0.5
        self.workspace = torch.zeros(binding.MPQ_CACHE_WORKSPACE, dtype=torch.uint8, device=DEV)

    def requests(self, B):
        i32 = lambda *a, **k: torch.tensor(*a, dtype=torch.int32, device=DEV)
        self.lens, self.table = i32([0] * B), torch.full((B, COLS), -1, dtype=torch.int32, device=DEV)
        self.pool, self.count = i32(list(range(PAGES))), i32([PAGES, 0])

    def tokens(self, x, add, after=lambda: None):
        """The new tokens x [N][d] of the requests into the cache: (their queries, slots, taken)."""
        slots, pos, taken = binding.mpq_pages_extend(add, self.lens, self.table, self.pool, self.count, PAGE, len(x))
        after()
        qkv = binding.mpq_g4_linear(x, self.w_in, self.in_layout)
        after()
        q, k, v = qkv.view(len(x), -1, DIM).split((HQ, H, H), 1)
        binding.mpq_rotate(q, k, pos, self.turns, norm=True, q_weight=self.q_weight, k_weight=self.k_weight, Yq=q, Yk=k)
        after()
        binding.mpq_cache_write(k, v, slots, self.cache, self.codes, self.scales)
        after()
        return q, k, v, slots, taken

    def step(self, x, add, after=lambda: None):
        q, *_ = self.tokens(x, add, after)
        o = binding.mpq_cache_attention(q, self.table, self.lens, self.cache, self.codes, self.scales,
                                        workspace=self.workspace)
        after()
        return binding.mpq_g4_linear(o.view(len(x), -1), self.w_out, self.out_layout)

    def state(self):
        return [t.clone() for t in (self.lens, self.table, self.count, self.pool, self.codes, self.scales)]

    def restore(self, saved):
        for t, s in zip((self.lens, self.table, self.count, self.pool, self.codes, self.scales), saved):
            t.copy_(s)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, False)])
def test_prompts_then_steps(gpu, group, zeros):
    layer = Layer(group, zeros)
    layer.requests(5)
    add = torch.tensor([40, 1, 0, 33, 100], dtype=torch.int32, device=DEV)
    N = int(add.sum()) + 10                                        # a padded batch
    x = layer.rand(N, D).to(layer.dtype)
    q, k, v, slots, taken = layer.tokens(x, add)
    assert taken.tolist() == add.tolist() and bool((slots[-10:] == -1).all())
    # what the cache holds is what was projected, within half a step of 8 bits (and the reading's rounding)
    K, V = binding.mpq_cache_read(slots[:-10], layer.cache, layer.codes, layer.scales, dtype=torch.float32)
    for got, part in ((K, k[:-10].float()), (V, v[:-10].float())):
        step = part.abs().amax(-1, keepdim=True) / 127
        assert bool(((got - part).abs() <= 0.501 * step).all())
    # the keys are the projection's, normed and turned by the requests' own positions
    raw = binding.mpq_g4_linear(x, layer.w_in, layer.in_layout).view(N, -1, DIM)[:, HQ:HQ + H]
    pos = np.concatenate([np.arange(n) for n in add.tolist()] + [np.zeros(10)])
    want, mag = ref.rotate(raw.double().cpu().numpy(), pos, layer.freq, True, layer.k_weight.double().cpu().numpy(),
                           1e-6, False)
    assert (np.abs(k.double().cpu().numpy() - want) <= 21 * 2.0 ** -24 * mag + 2.0 ** -8 * np.abs(want) * 1.001).all()
    # steps, each call waited for, and the same steps in one go and as a graph's replays
    one = torch.ones(5, dtype=torch.int32, device=DEV)
    xs = [layer.rand(5, D).to(layer.dtype) for _ in range(20)]
    before = layer.state()
    wanted = [layer.step(t, one, torch.cuda.synchronize) for t in xs]
    end = layer.state()
    layer.restore(before)
    got = [layer.step(t, one) for t in xs]
    assert all(torch.equal(a, b) for a, b in zip(got, wanted))
    assert all(torch.equal(a, b) for a, b in zip(layer.state()[:4], end[:4]))
    layer.restore(before)
    static = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(static, one)
    for t, w in zip(xs, wanted):
        static.copy_(t)
        graph.replay()
        assert torch.equal(y, w)
    assert all(torch.equal(a, b) for a, b in zip(layer.state()[:4], end[:4]))
    assert layer.lens.tolist() == [60, 21, 20, 53, 120]


def test_drafts_taken_back_and_a_full_pool(gpu):
    """Drafted tokens cut back and written again give the same step; a request without room leaves the others'
    outputs alone."""
    layer = Layer(64, True)
    layer.requests(3)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    layer.tokens(layer.rand(64, D).to(layer.dtype), i32([30, 15, 19]))
    one = torch.ones(3, dtype=torch.int32, device=DEV)
    x = layer.rand(3, D).to(layer.dtype)
    before = layer.state()
    want = layer.step(x, one)
    layer.restore(before)
    keep = layer.lens.clone()
    layer.tokens(layer.rand(15, D).to(layer.dtype), i32([5, 5, 5]))
    binding.mpq_pages_trim(keep, layer.lens, layer.table, layer.pool, layer.count, PAGE)
    assert torch.equal(layer.lens, keep) and torch.equal(layer.pool[:int(layer.count[0])], before[3][:int(before[2][0])])
    assert torch.equal(layer.step(x, one), want)
    # request 1 (16 tokens, a page) needs a page and finds none
    layer.restore(before)
    layer.tokens(layer.rand(1, D).to(layer.dtype), i32([0, 1, 0]))
    layer.count[0] = 0
    y = layer.step(x, one)
    assert layer.lens.tolist() == [31, 16, 20]
    assert torch.equal(y[0], want[0]) and torch.equal(y[2], want[2])
