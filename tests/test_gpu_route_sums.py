"""Sums of two ranks beyond fp32's range: groups masked by the lowest value of the type are open and come last, before closed ones only.  Choices are
exact; tolerances as in test_gpu_route."""
import numpy as np
import pytest

import test_gpu_route as R
from test_gpu_route import ctx  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("scores", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups", [(16, 4), (64, 8), (256, 8), (512, 16), (60, 4)])
def test_biases_of_the_largest_magnitude(ctx, E, groups, scores):  # noqa: F811
    rng = np.random.default_rng(E + scores)
    n, per = 200, E // groups
    of = np.arange(E) // per
    logits = rng.standard_normal((n, E))
    logits[:, of == 0] = -np.inf                                    # closed in every token, with the lowest number
    logits[::3, of != groups - 1] = -np.inf                         # only the last group is open
    for low, high in ((-MOST, -MOST), (-MOST, 0.0), (-MOST, MOST), (MOST, 0.0), (0.75 * MOST, 0.5 * MOST)):
        bias = np.where(of % 2 == (groups - 1) % 2, low, high).astype(np.float64)
        for top in (1, 2, groups - 1):
            R._run(ctx, logits, bias, rng.standard_normal((n, 3)), R.F32, 0, scores=scores, fan=3, groups=groups, top_groups=top, group_best=2)
