"""The evaluation operators at the ends of their ranges: alignments, magnitudes, counts, threads and what they refuse."""
import math
import threading

import pytest
import torch

import eval_reference as ref
from paper_2201_13096_b200 import binding, build as build_mod, evaluate
from test_evaluate import BF16, F16, F32, norm_bounds, rand

INF = math.inf
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


# ------------------------------------------------------------------------------------------------ layer norm

@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,D", [(7, 768), (5, 8), (300, 96)])
@pytest.mark.parametrize("lead", range(8))
def test_layer_norm_of_rows_that_start_anywhere_with_fp32_parameters(dtype, R, D, lead):
    """A row's first granule may begin before the row: the parameters are not read there."""
    x = rand(R, D, seed=1, dtype=dtype, pad=12 - lead, shift=lead)
    w, b = 1.0 + 0.2 * rand(D, seed=2), 0.3 * rand(D, seed=3)
    want, mean64, rstd64 = ref.layer_norm(x, w, b, 1e-5)
    y, mean, rstd = evaluate.layer_norm(x, w, b)
    ref.close(y, want, norm_bounds(x, w, b, want, rstd64), "y")
