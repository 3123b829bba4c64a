"""The example that runs CCD++, the softmax loss over all items and gradient clipping together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_choices_get_likelier():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "choose_items.py")
    spec = importlib.util.spec_from_file_location("choose_items", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last = m.main(["--users", "800", "--items", "500", "--ratings", "30000", "--k", "16", "--steps", "60", "--batch", "256"])
    assert last < first
