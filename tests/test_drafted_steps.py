"""The operators of a drafted step together, as a server uses them: append, bounds, selection or shared prefix, attention, verification (GPU)."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("dim,heads,drafts", [(128, (32, 8), 4), (64, (8, 4), 3), (128, (8, 1), 0), (64, (8, 1), 7)])
def test_steps_hold_to_the_definitions(dim, heads, drafts):
    spec = importlib.util.spec_from_file_location("drafted_steps", os.path.join(ROOT, "examples", "drafted_steps.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    got = m.run(sequences=5, described=420, steps=6, drafts=drafts, budget=12, dim=dim, heads=heads, seed=dim + drafts)
    assert got["error_of_bound"] <= 1 and got["emitted"] >= 5 * 6
