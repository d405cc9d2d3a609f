"""What building needs, and when (no GPU, no compiler): nothing where nothing is stale."""
import pytest

from paper_2002_09049_gb300 import _build


def test_nothing_stale_needs_no_toolkit(monkeypatch):
    def missing():
        raise RuntimeError("nvcc not found")

    monkeypatch.setattr(_build, "nvcc", missing)
    monkeypatch.setattr(_build, "up_to_date", lambda lib=None: True)
    monkeypatch.setattr(_build, "_binding_up_to_date", lambda: True)
    assert _build.build() == _build.LIB and _build.build(checked=True) == _build.CHECKED_LIB
    monkeypatch.setattr(_build, "up_to_date", lambda lib=None: False)
    with pytest.raises(RuntimeError, match="nvcc"):
        _build.build()
