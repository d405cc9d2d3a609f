"""A serving call that has to wait for room in its stream's queue lets other Python threads run."""
import threading
import time

import pytest
import torch

from paper_2002_09049_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_other_threads_run_while_a_launch_waits(gpu):
    lay = binding.mpq_mx_layout(4, 64)
    x = torch.randn(4, 64, device=DEV)
    packed = binding.mpq_mx_quantize(x, lay)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    torch.cuda._sleep(10_000_000)
    end.record()
    torch.cuda.synchronize()
    a_second = int(10_000_000 * 1000 / begin.elapsed_time(end))
    stop, longest = threading.Event(), [0.0]

    def tick():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.002)
            now = time.perf_counter()
            longest[0], last = max(longest[0], now - last), now

    t = threading.Thread(target=tick)
    t.start()
    torch.cuda._sleep(a_second)
    start = time.perf_counter()
    for _ in range(6000):                # far more than a queue holds
        binding.mpq_mx_quantize(x, lay, packed)
    took = time.perf_counter() - start
    stop.set()
    t.join()
    torch.cuda.synchronize()
    assert took > 0.5                    # (a launch did wait)
    assert longest[0] < 0.25
