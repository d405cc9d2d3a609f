"""The ways in which the attention over the cache cuts its work, by the number of sequences and the lengths of
their rows: a warp a row, a CTA a row, ranges of any rows; one sequence a lane, one a thread or several.
Against 64-bit sums with the bounds of test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from test_gpu_cache import Scene

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def ragged(n, top, seed, empty=0.2):
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, top, n)
    lens[rng.random(n) < empty] = 0
    return [int(v) for v in lens]


@pytest.mark.parametrize("lens,heads,group,dim,bits", [
    ([64] * 24, 8, 2, 64, 8),                         # up to 32 sequences, more rows than CTAs: a warp a row
    (ragged(32, 90, 1), 8, 3, 64, 4),
    (ragged(30, 60, 2), 8, 1, 128, 8),
    (ragged(32, 60, 3, 0.0), 6, 10, 256, 8),
    ([80] * 200, 1, 4, 128, 8),                       # the same, a sequence a thread
    (ragged(1200, 60, 4), 1, 2, 64, 8),               # several sequences a thread, some of them empty
    ([64] * 1000, 2, 1, 64, 8),
    (ragged(520, 70, 5), 1, 9, 256, 8),
    (ragged(1100, 40, 6), 3, 1, 64, 4),               # more rows than warps
    ([0] * 800, 2, 2, 64, 8)])
def test_batches(gpu, lens, heads, group, dim, bits):
    s = Scene(lens, heads, group, dim, bits, 16, "fp16", len(lens) + dim, loud=2.0)
    o, lse = s.run()
    s.check(o, lse)


@pytest.mark.parametrize("n,at", [(513, 0), (700, 300), (1030, 1029)])
def test_one_long_row_among_many(gpu, n, at):
    """Several CTAs share it, wherever its thread's other sequences stand."""
    lens = ragged(n, 30, n)
    lens[at] = 9000
    s = Scene(lens, 1, 2, 64, 8, 32, "bf16", n, loud=2.0)
    o, lse = s.run()
    s.check(o, lse)
    for _ in range(2):
        again = s.run()
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_few_live_among_many(gpu):
    """A CTA a row where only a few of many sequences have any tokens."""
    lens = [0] * 900
    for b in range(0, 900, 9):
        lens[b] = 200
    s = Scene(lens, 1, 4, 64, 8, 16, "bf16", 3, loud=2.0)
    o, lse = s.run()
    s.check(o, lse)


def test_short_rows_are_not_cut(gpu):
    """1,000 sequences of 64 tokens, two key heads: a warp a row, as in batches of 250, so the same bits."""
    s = Scene([64] * 1000, 2, 2, 64, 8, 16, "bf16", 7, loud=2.0)
    o, lse = s.run()
    q, table = s.q, s.table
    for i in range(0, 1000, 250):
        s.q, s.table, s.lens = q[i:i + 250], table[i:i + 250], [64] * 250
        part, part_lse = s.run()
        assert torch.equal(o[i:i + 250], part) and torch.equal(lse[i:i + 250], part_lse)
