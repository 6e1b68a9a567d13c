"""Padded tokens (all logits -infinity) beside tokens whose ranks are too near to each other for fp32: choices of -1 and gates of 0 in every place.
Choices are exact; tolerances as in test_gpu_route."""
import numpy as np
import pytest

import test_gpu_route as R
from test_gpu_route import ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [R.F32, R.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("scores", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [True, False], ids=["bias", ""])
@pytest.mark.parametrize("E,groups,top,best", [(8, 1, 1, 1), (16, 1, 1, 1), (60, 1, 1, 1), (64, 8, 4, 2), (256, 1, 1, 1), (256, 8, 4, 2), (512, 1, 1, 1)])
def test_padding_beside_near_ranks(ctx, E, groups, top, best, with_bias, scores, renormalise, dtype):  # noqa: F811
    rng = np.random.default_rng(E + groups)
    n = 129
    logits, bias = rng.standard_normal((n, E)), 0.1 * rng.standard_normal(E).astype(np.float32)
    pair = rng.permutation(E)[:2]
    logits[:, pair] = 3.0                                           # equal scores, biases a step of fp32 apart: only 64 bits tell which is first
    bias[pair] = 0.5, np.nextafter(np.float32(0.5), np.float32(1))
    logits[rng.random(n) < 0.6] = -np.inf
    assert np.isneginf(logits).all(1).any() and not np.isneginf(logits).all(1).all()
    for fan in (1, 2, 3, 6):
        choice = R._run(ctx, logits, bias if with_bias else None, rng.standard_normal((n, fan)), dtype, 0, scores=scores, fan=fan, groups=groups, top_groups=top,
                        group_best=best, renormalise=renormalise)
        assert (choice[np.isneginf(logits).all(1)] == -1).all()
