"""The example that runs the search with the evaluation operators, end to end."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_search_over_a_stitched_model_and_its_tuning():
    import stitched_search

    out = stitched_search.main(["--trials", "12", "--tune-steps", "6"])
    assert abs(out["dense"]) < 1e-4                      # the dense model is its own teacher
    assert out["time"] <= out["budget"] and out["evals"] >= 13
    assert 0 < out["searched"] < out["uniform"] * 1.05   # a searched profile is not worse than one sparsity for all
    assert out["tuned"] < out["searched"]
    assert out["tuning"][0] == pytest.approx(out["searched"], rel=1e-3) and out["tuning"][-1] < out["tuning"][0]
