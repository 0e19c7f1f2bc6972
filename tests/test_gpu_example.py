"""The example that learns a head from a teacher, lays it out in 8 bits and draws from it."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "head_from_teacher.py")


def test_learns_draws_and_finds_its_phrases():
    spec = importlib.util.spec_from_file_location("head_from_teacher", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main()
    assert r["losses"][-1] < 0.5 * r["losses"][0] and np.isfinite(r["losses"]).all()
    assert (r["best"] == r["teacher"]).mean() > 0.8
    assert (r["tokens"][:, 1:] >= 0).all() and (r["tokens"] < 2000).all()
    assert (r["probs"] > 0).all() and (r["probs"] <= 1).all()
    # The second answer begins as the first one did, so it meets the phrases taken from it.
    assert r["hits"] >= 16
    again = m.main()
    assert (again["tokens"] == r["tokens"]).all() and (again["probs"] == r["probs"]).all()
