"""examples/distill_drafter.py end to end: the training lowers the divergence, and the round accepts more of what the drafter drafts."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_the_drafter_learns(gpu):
    print("[case] example distill_drafter", flush=True)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_drafter.py")
    spec = importlib.util.spec_from_file_location("distill_drafter", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.main(steps=60, verbose=False)
    assert r["loss"][1] < 0.7 * r["loss"][0]
    assert r["expected"][1] > r["expected"][0]
    assert r["accepted"][1] > r["accepted"][0]
