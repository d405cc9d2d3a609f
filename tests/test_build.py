"""What building needs, and when (no GPU, no compiler): nothing where nothing is stale."""
import pytest
import torch

from paper_2002_09049_gb300 import _build, binding


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


def test_extension_of_another_torch_is_neither_kept_nor_loaded(monkeypatch):
    _build.build()
    assert _build.binding_fits() and _build._binding_up_to_date()
    monkeypatch.setattr(torch, "__version__", "1.0")
    assert not _build._binding_up_to_date()
    with pytest.raises(RuntimeError, match="another Python or torch"):
        binding._Unloaded().mx_quantize
    monkeypatch.undo()
    monkeypatch.setattr(_build.sysconfig, "get_config_var", lambda name: "cpython-2-none")
    assert not _build._binding_up_to_date()
