"""Where operands may lie (no GPU): no kernel loads with a cluster multicast, whose source has to be this
GPU's own memory, which nothing can promise of a pointer that a caller gives."""
import glob
import os
import re

from paper_2002_09049_gb300 import _build


def _instructions(path):
    """The PTX instructions in a source's string literals, neighbouring literals joined."""
    with open(path) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for run in re.findall(r'"(?:[^"\\]|\\.)*"(?:\s*"(?:[^"\\]|\\.)*")*', text):
        joined = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', run))
        yield from joined.split(";")


def test_no_multicast_loads():
    paths = [p for e in ("cu", "cuh", "cpp") for p in
             glob.glob(os.path.join(_build.CSRC, "**", f"*.{e}"), recursive=True)]
    copies = [(os.path.basename(p), i) for p in paths for i in _instructions(p) if "cp.async.bulk" in i]
    assert copies                                       # (the scan sees the tile copies)
    assert not [c for c in copies if "multicast" in c[1]]
