"""The example that trains a next-item model and serves it: its loss falls, and items served one by one from the kept
states score as they do in one call over the whole history."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype,bar", [("f32", 1e-4), ("bf16", 4e-2)])
def test_example(monkeypatch, dtype, bar):
    """Bars: the outputs of the layer differ by roundings of their type (2^-8 in bf16), which the projections and the
    products with the item table carry on, a few of them one behind the other."""
    monkeypatch.syspath_prepend(os.path.join(ROOT, "examples"))
    monkeypatch.setattr(sys, "argv", ["next_item.py", "--steps", "30", "--dtype", dtype])
    import next_item
    losses, far = next_item.main()
    assert losses[-1] < 0.8 * losses[0]
    assert far < bar
