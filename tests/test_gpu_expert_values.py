"""Products and factors of experts: values that are not finite.  (Sums against float64: test_gpu_experts.py.)"""
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


def _randn(g, *shape):
    return torch.randn(*shape, generator=g).cuda()


# Every tile of the contractions over rows: 64 x 64 with four and with two groups of waves, 128 x 128, operands straight to LDS.
@pytest.mark.parametrize("E,ci,co,dtype", [(4, 61, 100, F32), (40, 131, 139, F32), (64, 100, 127, F32), (4, 61, 100, BF16), (40, 131, 139, BF16),
                                           (64, 100, 127, BF16), (4, 64, 96, BF16), (3, 264, 272, BF16)])
def test_one_channel_that_is_not_finite(E, ci, co, dtype):
    """An infinity in dy[:, o] and a NaN in x[:, k] reach what is formed from these channels; all other sums, those of the bias among
    them, keep the bits they have without."""
    g = torch.Generator()
    g.manual_seed(E + ci)
    n = 6 * E
    layer = wl.fc_layer(1, ci, co, 1)
    ctx = kfac.Context([layer], workspace_bytes=kfac.kfac_expert_workspace_bytes(layer, E, n))
    x, dy = _randn(g, n, ci).to(dtype), _randn(g, n, co).to(dtype)
    offsets = (torch.arange(E + 1, dtype=torch.int32) * 6).cuda()

    def run():
        dW = torch.full((E, co, ci + 1), 5.0, device="cuda")
        A, G = torch.full((E, ci + 1, ci + 1), 5.0, device="cuda"), torch.full((E, co, co), 5.0, device="cuda")
        kfac.kfac_expert_grad_weight(ctx, layer, None, offsets, x, dy, dW)
        kfac.kfac_stats_expert(ctx, layer, None, offsets, x, dy, 0.0, A, G)
        torch.cuda.synchronize()
        return dW, A, G

    clean = run()
    assert all(bool(torch.isfinite(t).all()) for t in clean)
    for e, o, k in ((0, 5, 3), (E - 1, co - 1, ci - 1), (E // 2, 18, 50)):
        row = 6 * e + 4
        old = x[row, k].item(), dy[row, o].item()
        x[row, k], dy[row, o] = float("nan"), float("inf")
        got = run()
        x[row, k], dy[row, o] = old
        hit = [torch.zeros(t.shape, dtype=torch.bool) for t in clean]
        hit[0][e, o], hit[0][e, :, k] = True, True
        hit[1][e, k], hit[1][e, :, k] = True, True
        hit[2][e, o], hit[2][e, :, o] = True, True
        for name, a, b, h in zip(("dW", "A", "G"), got, clean, hit):
            a, b = a.cpu(), b.cpu()
            assert torch.equal(a[~h], b[~h]), "%s: %d values of other channels" % (name, int((a[~h] != b[~h]).sum()))
            assert not bool(torch.isfinite(a[h]).any()), name
    ctx.close()
