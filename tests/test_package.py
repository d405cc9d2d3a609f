"""What the package offers by name (no GPU needed)."""
import inspect

import paper_2002_09049_gb300 as package
from paper_2002_09049_gb300 import binding

# what a program asks of a run rather than of its data, and the test hooks, stay in `binding`
OF_A_RUN = {"mpq_build_options", "mpq_device_status", "mpq_last_error", "mpq_set_wait_limit"}


def test_every_operator_is_offered():
    names = {n for n, f in inspect.getmembers(binding) if n.startswith("mpq_") and callable(f)}
    assert {"mpq_g4_linear", "mpq_rotate", "mpq_pages_extend", "mpq_cache_attention"} <= names
    missing = {n for n in names - OF_A_RUN if not n.startswith("mpq_test_") and not hasattr(package, n)}
    assert not missing
