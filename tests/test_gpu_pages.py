"""The pages of a cache's requests on the GPU: every output, table entry and pool entry equal to those of the
same steps taken one request after another on the host."""
import numpy as np
import pytest
import torch

import _decode_step as ref
from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
t32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


class State:
    """Requests with pages of their own (numbers that are no permutation of a range), on both sides."""

    def __init__(self, rng, lens, cols, page, spare, room=0):
        self.page, self.lens = page, np.array(lens, np.int32)
        held = [max(0, min(-(-int(n) // page), cols)) for n in lens]
        order = (rng.permutation(sum(held) + spare + 5) * 3 + 1).astype(np.int32)
        self.table = np.full((len(lens), cols), -7, np.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.pool = np.concatenate([order[at:at + spare], np.full(sum(held) + room, -9, np.int32)]).astype(np.int32)
        self.count = spare
        self.dev = dict(lens=t32(self.lens), table=t32(self.table.reshape(len(lens), cols)), pool=t32(self.pool),
                        count=t32([spare, 0]))

    def extend(self, add, N, in_place=True, count=None):
        add, d = np.asarray(add, np.int32), self.dev
        out = {} if in_place else dict(new_lens=torch.full_like(d["lens"], 77), new_count=torch.full_like(d["count"], 77))
        got = binding.mpq_pages_extend(t32(add), d["lens"], d["table"], d["pool"], d["count"], self.page, N, **out)
        slots, pos, taken, self.table, lens, count = ref.extend(add, self.lens, self.table, self.pool, self.count,
                                                                self.page, N)
        for g, w in zip(got, (slots, pos, taken)):
            assert np.array_equal(g.cpu().numpy(), w)
        self.after(lens, count, out)
        return slots, pos, taken

    def trim(self, keep, in_place=True):
        keep, d = np.asarray(keep, np.int32), self.dev
        out = {} if in_place else dict(new_lens=torch.full_like(d["lens"], 77), new_count=torch.full_like(d["count"], 77))
        binding.mpq_pages_trim(t32(keep), d["lens"], d["table"], d["pool"], d["count"], self.page, **out)
        lens, self.pool, count = ref.trim(keep, self.lens, self.table, self.pool, self.count, self.page)
        self.after(lens, count, out)

    def after(self, lens, count, out):
        d = self.dev
        if out:                                     # the state of before is still there
            assert np.array_equal(d["lens"].cpu().numpy(), self.lens)
            assert d["count"].tolist() == [self.count, 0]
            d["lens"], d["count"] = out["new_lens"], out["new_count"]
        self.lens, self.count = lens, count
        assert np.array_equal(d["lens"].cpu().numpy(), lens)
        assert d["count"].tolist() == [count, 0]
        assert np.array_equal(d["table"].cpu().numpy(), self.table)
        assert np.array_equal(d["pool"].cpu().numpy(), self.pool)


def sizes(rng, B, most):
    n = np.exp(rng.uniform(0, np.log(most + 1), B)).astype(np.int64)
    n[rng.random(B) < 0.15] = 0
    return n


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
@pytest.mark.parametrize("B,longest,most", [(1, 40, 1), (1, 1, 500), (5, 100, 9), (33, 300, 70), (257, 50, 30),
                                            (1025, 90, 12), (3000, 30, 4), (9, 3000, 5000)])
def test_a_run_of_steps(gpu, B, longest, most, page, in_place):
    """Admitted, extended and cut back in turn, with room for all, for some and for none."""
    rng = np.random.default_rng(B * 100 + page)
    lens = sizes(rng, B, longest)
    cols = -(-(longest + most) // page)
    need = int((-(-(lens + most) // page)).sum())
    s = State(rng, lens, cols, page, max(1, need // 3))
    for turn in range(4):
        add = sizes(rng, B, most)
        N = int(add.sum()) + (0, 64, -3, 5)[turn]
        s.extend(add, max(N, 0), in_place)
        s.trim(np.where(rng.random(B) < 0.4, 0, s.lens - rng.integers(-2, 6, B)), in_place)
        s.extend(np.ones(B), B, in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_limits(gpu, in_place):
    """Nothing asked, negative lengths and additions, full tables, counts past the pool or below zero."""
    rng = np.random.default_rng(1)
    s = State(rng, [0, 16, 17, -4, 48, 47, 3, 500], 3, 16, 4, room=2)
    s.extend([0, 0, 0, 5, 1, 2, -9, 1], 40, in_place)
    s.extend([0] * 8, 0, in_place)
    s.extend([2 ** 31 - 1, 1, 1, 1, 1, 1, 1, 1], 100, in_place)
    s.extend([40, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1, 1, 1, 1], 100, in_place)
    s.extend([1, 1, 1, -1, -1, 1, -2 ** 31, 1], 6, in_place)
    s.trim([-5, 2 ** 31 - 1, 16, 3, 0, 1, 2, 10], in_place)
    for count in (1000, -3):
        s.count = count
        s.dev["count"][0] = count
        if in_place:
            s.extend([9] * 8, 100)
            s.count = min(max(s.count, 0), len(s.pool))


@pytest.mark.parametrize("B,cols,N", [(0, 3, 5), (4, 0, 7), (0, 0, 0), (3, 2, 0)])
def test_no_requests_no_columns_no_room(gpu, B, cols, N):
    s = State(np.random.default_rng(2), [0] * B, cols, 16, 3)
    s.extend([1, 0, 2, 1][:B], N)
    s.trim([0] * B)


def test_a_step_taken_back_leaves_the_state(gpu):
    s = State(np.random.default_rng(3), [5, 100, 0, 31], 9, 16, 11)
    pool, lens = s.pool.copy(), s.lens.copy()
    s.extend([30, 1, 17, 1], 64)
    s.trim(lens)
    assert np.array_equal(s.pool, pool) and np.array_equal(s.lens, lens) and s.count == 11


def test_long_requests_and_many_tokens(gpu):
    """Several CTAs' tokens, requests of up to 2^20 tokens; the largest number of requests."""
    rng = np.random.default_rng(4)
    s = State(rng, [0, 1 << 20, 5], (1 << 21) // 64 + 1, 64, 40000)
    s.extend([1 << 20, 300001, 1 << 19], (1 << 21) + 77)
    s.trim([0, 1 << 20, 5])
    B = binding.MPQ_PAGES_MAX_REQUESTS
    s = State(rng, rng.integers(0, 40, B), 4, 16, B)
    for in_place in (True, False):
        s.extend(rng.integers(0, 3, B), 2 * B, in_place)
        s.trim(s.lens - rng.integers(0, 20, B), in_place)


def test_slots_past_32_bits(gpu):
    """A slot is a page times its size in 64 bits; a negative page is no slot."""
    add, lens = t32([3, 1, 1]), t32([0, 16, 5])
    table = t32([[0, 0], [5, 0], [-1, 0]])
    pool, count = t32([1 << 30, 2 ** 31 - 1]), t32([2, 0])
    slots, _, taken = binding.mpq_pages_extend(add, lens, table, pool, count, 16, 5)
    base = (2 ** 31 - 1) * 16
    assert slots.tolist() == [base, base + 1, base + 2, (1 << 30) * 16, -1] and taken.tolist() == [3, 1, 1]


def test_stream_and_graph(gpu):
    """A captured extension and cut: every replay is a step on the state it finds."""
    rng = np.random.default_rng(5)
    s, d = State(rng, [10, 0, 40], 8, 16, 12), None
    d = s.dev
    add, keep = t32([1, 17, 2]), t32([2 ** 31 - 1, 3, 2 ** 31 - 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slots, pos, taken = binding.mpq_pages_extend(add, d["lens"], d["table"], d["pool"], d["count"], 16, 20)
        binding.mpq_pages_trim(keep, d["lens"], d["table"], d["pool"], d["count"], 16)
    for _ in range(6):
        graph.replay()
        w = ref.extend(add.cpu().numpy(), s.lens, s.table, s.pool, s.count, 16, 20)
        for g, x in zip((slots, pos, taken, d["table"]), w):
            assert np.array_equal(g.cpu().numpy(), x)
        s.table = w[3]
        s.lens, s.pool, s.count = ref.trim(keep.cpu().numpy(), w[4], s.table, s.pool, w[5], 16)
        assert d["count"].tolist() == [s.count, 0] and np.array_equal(d["lens"].cpu().numpy(), s.lens)
        assert np.array_equal(d["pool"].cpu().numpy(), s.pool)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = binding.mpq_pages_extend(add, d["lens"], d["table"], d["pool"], d["count"], 16, 20, stream=side)
    side.synchronize()
    w = ref.extend(add.cpu().numpy(), s.lens, s.table, s.pool, s.count, 16, 20)
    assert all(np.array_equal(g.cpu().numpy(), x) for g, x in zip(got, w))


def test_refusals(gpu):
    mk = lambda: [t32([1, 1]), t32([0, 0]), t32([[0], [0]]), t32([3, 4, 5]), t32([3, 0])]
    def both(i, bad, error):
        for f in (lambda a: binding.mpq_pages_extend(*a, 16, 2), lambda a: binding.mpq_pages_trim(*a, 16)):
            a = mk()
            a[i] = bad
            with pytest.raises(error):
                f(a)
    for i in range(5):
        both(i, mk()[i].long(), TypeError)
        both(i, mk()[i].cpu(), ValueError)
    both(1, t32([0]), ValueError)
    both(2, t32([[0]]), ValueError)
    both(2, t32([0, 0]), ValueError)
    both(2, torch.zeros(2, 4, dtype=torch.int32, device=DEV)[:, ::2], ValueError)
    both(4, t32([3]), ValueError)
    a = mk()
    with pytest.raises(binding.MPQError):
        binding.mpq_pages_extend(*a, 16, 2, taken=a[0])                # an output over an input
    with pytest.raises(ValueError):
        binding.mpq_pages_extend(*a, 16, -1)
    with pytest.raises(binding.MPQError):
        binding.mpq_pages_extend(*a, 0, 2)
    with pytest.raises(TypeError):
        binding.mpq_pages_extend(*a, 16, 2, slots=torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        binding.mpq_pages_extend(*a, 16, 2, new_lens=t32([1, 2, 3]))
