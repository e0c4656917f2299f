"""The serving example runs and its own checks (against plain torch arithmetic) hold, at its sizes and at odd ones."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kw", [{}, dict(layers=1, sequences=1, prompt=33, steps=1, budget=20, window=7, sinks=0, heads=6, kv_heads=2)])
def test_kv_serving(kw):
    spec = importlib.util.spec_from_file_location("kv_serving", os.path.join(ROOT, "examples", "kv_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    if "budget" in kw:  # 32 recent tokens are the example's; a smaller budget is refused by the call
        with pytest.raises(Exception):
            m.main(**kw, quiet=True)
        kw = dict(kw, budget=34)
    assert 0 < m.main(**kw, quiet=True) <= 1.0001
