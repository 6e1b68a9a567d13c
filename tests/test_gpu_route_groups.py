"""Groups of experts whose two best ranks take most of each other away: their order is that of the sums in 64 bits.  Choices are exact; tolerances
as in test_gpu_route."""
import numpy as np
import pytest

import test_gpu_route as R
from test_gpu_route import ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scores", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [1.0, 100.0, 1024.0, 65536.0])
@pytest.mark.parametrize("E,groups", [(16, 8), (32, 16), (64, 8), (256, 8), (512, 16)])
def test_sums_of_ranks_of_opposite_sign(ctx, E, groups, size, scores):  # noqa: F811
    """Two open experts a group, with biases b and -b: the sum is that of their scores, b's size goes into the rounding of each rank.  Groups come in
    pairs whose scores differ by a few 2^-21, and an odd number of groups takes part."""
    rng = np.random.default_rng(E + int(size) + scores)
    n, per, step = 800, E // groups, np.spacing(np.float32(size))
    b = size + step * rng.permutation(64)[:groups]                  # (exact in fp32)
    bias = np.full(E, -np.inf)
    bias[::per], bias[1::per] = b, -b
    logits = rng.standard_normal((n, groups, per)).astype(np.float32)
    logits[:, :, 2:] = -np.inf                                      # (so that the two have all of a softmax)
    logits[:, 1::2] = logits[:, ::2]
    logits[:, 1::2, 0] += np.float32(2.0 ** -21) * rng.choice([-3, -2, -1, 1, 2, 3], (n, groups // 2))
    logits = logits.reshape(n, E)
    # no two sums that 64 bits leave open: the ranks' roundings there are within 2^-53 of the size, four of them
    s = R.B.scores(logits.astype(np.float64), scores == 1)[:, np.isfinite(bias)].reshape(n, groups, 2).sum(2)
    sums = np.sort(s, 1)
    assert (np.diff(sums, axis=1) > 16 * 2.0 ** -53 * size).all()
    for top in (1, 3, groups - 1):
        R._run(ctx, logits, bias, rng.standard_normal((n, 2)), R.F32, 0, scores=scores, fan=2, groups=groups, top_groups=top, group_best=2)
