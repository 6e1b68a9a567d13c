"""Experts in a context created with fp32_products = KFAC_PRODUCTS_FP32_MFMA: the parity cases once more, to the same tolerances, and
what the fp32 matrix instruction does that the planes of the default mode do not."""
import numpy as np
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl
import test_gpu_experts as X
from test_gpu_expert_values import test_one_channel_that_is_not_finite  # noqa: F401

pytestmark = pytest.mark.gpu

gpu = X.gpu


@pytest.fixture(autouse=True)
def fp32_instruction_mode():
    with kfac.default_options(fp32_products=kfac.KFAC_PRODUCTS_FP32_MFMA):   # for every context the tests create
        yield


# re-collected here, so that they run with the fixture above
test_forward_and_gradients = X.test_forward_and_gradients
test_factors = X.test_factors
test_nan_stays_where_it_is = X.test_nan_stays_where_it_is
test_sorted_choices_need_no_order = X.test_sorted_choices_need_no_order
test_gradients_by_differences = X.test_gradients_by_differences
test_many_tiles = X.test_many_tiles
test_rows_of_all_lengths_of_a_contraction = X.test_rows_of_all_lengths_of_a_contraction
test_captured_in_a_graph = X.test_captured_in_a_graph


def _outputs(c):
    y, dx = torch.empty(c.n, c.co, device="cuda"), torch.empty(c.n, c.ci, device="cuda")
    dW, A, G = (torch.empty(c.E, a, b, device="cuda") for a, b in ((c.co, c.ci + c.bias), (c.ci + c.bias, c.ci + c.bias), (c.co, c.co)))
    kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, c.x, c.W, y)
    kfac.kfac_expert_grad_input(c.ctx, c.layer, c.order, c.offsets, c.dy, c.W, dx)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW)
    kfac.kfac_stats_expert(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, 0.0, A, G)
    torch.cuda.synchronize()
    return y, dx, dW, A, G


# tiles of 64 x 64 with four groups of waves in the contractions over rows, with two, and of 128 x 128
SIZES = [(4, 61, 100), (40, 131, 139), (64, 100, 127)]


@pytest.mark.parametrize("E,ci,co", SIZES)
def test_an_infinity_stays_one(E, ci, co):
    """One infinite element of x and one of dy: infinities in what it reaches, which the planes make NaN."""
    c = X.Case(6 * E, 1, E, ci, co, 1, X.F32, "even")
    choice = torch.arange(6 * E, dtype=torch.int32) // 6
    kfac.kfac_segments(c.ctx, choice.cuda(), E, c.order, c.offsets)
    row, e, inf = 9, 1, float("inf")
    c.x[row, 7], c.dy[row, 11] = inf, -inf
    y, dx, dW, A, G = _outputs(c)
    assert torch.equal(y[row], inf * c.W[e, :, 7].sign()) and torch.equal(dx[row], -inf * c.W[e, 11, :ci].sign())
    others = torch.arange(ci, device="cuda") != 7
    assert torch.equal(dW[e, :, 7][torch.arange(co) != 11], inf * c.dy[row][torch.arange(co) != 11].sign())
    assert torch.equal(dW[e, 11, :ci][others], -inf * c.x[row][others].sign()) and float(dW[e, 11, ci]) == -inf
    assert torch.equal(A[e, 7, :ci], inf * c.x[row].sign()) and float(A[e, 7, ci]) == inf and float(A[e, ci, 7]) == inf
    assert torch.equal(G[e, 11], -inf * c.dy[row].sign())
    c.ctx.close()


@pytest.mark.parametrize("E,ci,co", SIZES)
def test_small_operands_keep_their_bits(E, ci, co):
    """x of 2^-120 against operands of one, where the planes lose the bits below 2^-133: the error is that of the sums.  All positive, so
    that no operand, product or sum is a subnormal."""
    c = X.Case(6 * E, 1, E, ci, co, 1, X.F32, "even")
    for t in (c.x, c.dy, c.W):
        t.copy_(1.0 + t.abs().remainder(1.0))
    c.x.mul_(2.0 ** -120)
    c.W[:, :, ci] = 0.0
    x, dy, W = X._values(c.x), X._values(c.dy), X._values(c.W)
    y, _, dW, _, _ = _outputs(c)
    for got, (ref, mag), m in ((y, X.T.expert_forward(c.choice, x, W, ci, 1, 1), ci + 1),
                               (dW[:, :, :ci], X.T.expert_grad_weight(c.choice, x, dy, E, 0, 1), c.longest)):
        assert np.all(np.abs(X._values(got) - ref) <= (m + 8) * 2.0 ** -24 * mag)
    c.ctx.close()


def test_bf16_is_the_same_in_both_modes():
    c = X.Case(70, 1, 3, 61, 33, 1, X.BF16, "even")
    y, z = torch.empty(70, 33, dtype=X.BF16, device="cuda"), torch.empty(70, 33, dtype=X.BF16, device="cuda")
    kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, c.x, c.W, y)
    with kfac.default_options(fp32_products=kfac.KFAC_PRODUCTS_SPLIT_BF16):
        other = kfac.Context([c.layer])
    kfac.kfac_expert_forward(other, c.layer, c.order, c.offsets, c.x, c.W, z)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    other.close()
    c.ctx.close()
