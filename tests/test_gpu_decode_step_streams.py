"""4-bit integer weights, rotation and page tables on several streams, from several threads and as several graphs at
once: every result is that of the call made alone."""
import threading

import numpy as np
import pytest
import torch

from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Work:
    """One chain of calls on tensors of its own: pages, layers of few and of many tokens (odd rows of x among
    them), a rotation."""

    def __init__(self, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
        self.lay = binding.mpq_g4_layout(640, 643, 32, True)
        self.w = binding.mpq_g4_quantize(0.05 * rand(640, 643), self.lay)
        self.x = [rand(T, 643).to(torch.bfloat16) for T in (3, 60, 200, 700)]
        self.turns = binding.mpq_rotation(10000.0 ** (-np.arange(0, 64, 2) / 64), DEV)
        self.pos = torch.randint(0, 9999, (700,), generator=gen, device=DEV, dtype=torch.int32)
        i32 = lambda *a: torch.tensor(*a, dtype=torch.int32, device=DEV)
        self.add, self.lens = i32([30, 0, 5, seed]), i32([7, 16, 0, 40])
        self.table = torch.arange(32, device=DEV, dtype=torch.int32).view(4, 8).contiguous()
        self.pool, self.count = torch.arange(40, device=DEV, dtype=torch.int32) + 100, i32([40, 0])

    def run(self):
        out = list(binding.mpq_pages_extend(self.add, self.lens, self.table, self.pool, self.count, 16, 64,
                                            new_lens=torch.empty_like(self.lens), new_count=torch.empty_like(self.count)))
        for x in self.x:
            y = binding.mpq_g4_linear(x, self.w, self.lay)
            out.append(y)
            out += binding.mpq_rotate(y.view(len(x), 10, 64)[:, :8], y.view(len(x), 10, 64)[:, 8:], self.pos[:len(x)],
                                      self.turns, norm=True)
        return out


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_streams_and_threads(gpu):
    works = [Work(i) for i in range(4)]
    want = [w.run() for w in works]
    torch.cuda.synchronize()
    bad = []

    def go(w, r):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for _ in range(15):
                got = w.run()
                side.synchronize()
                if not same(got, r):
                    bad.append(w)
    threads = [threading.Thread(target=go, args=a) for a in zip(works, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad and binding.mpq_device_status() == 0


def test_graphs_replayed_at_once(gpu):
    works = [Work(i) for i in range(3)]
    want = [w.run() for w in works]
    torch.cuda.synchronize()
    graphs = []
    for w in works:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = w.run()
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(10):
        for g, out, s in graphs:
            with torch.cuda.stream(s):
                for t in out:
                    t.zero_()
                g.replay()
        torch.cuda.synchronize()
        assert all(same(out, r) for (_, out, _), r in zip(graphs, want))


def test_the_current_device_and_stream_arguments(gpu):
    """A call with a stream argument runs there, and its outputs belong to it."""
    w = Work(9)
    want = w.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for x, r in zip(w.x, (want[3], want[6], want[9], want[12])):
        got = binding.mpq_g4_linear(x, w.w, w.lay, stream=side)
        side.synchronize()
        assert torch.equal(got, r)
