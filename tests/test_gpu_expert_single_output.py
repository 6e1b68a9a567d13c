"""Experts with one output channel: the distance of W's rows is that of the experts, whatever the strides of length-one dimensions say."""
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,ci", [(4, 40), (3, 1), (1, 24)])
def test_weights_of_one_row(dtype, E, ci):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    n = 30
    layer = wl.fc_layer(1, ci, 1, 0)
    g = torch.Generator()
    g.manual_seed(ci)
    x, W = torch.randn(n, ci, generator=g).cuda().to(dtype), torch.randn(E, 1, ci, generator=g).cuda().to(dtype)
    offsets = (torch.arange(E + 1) * n // E).int().cuda()
    ctx = kfac.Context([layer], workspace_bytes=kfac.kfac_expert_workspace_bytes(layer, E, n))
    want = torch.empty(n, 1, dtype=dtype, device="cuda")
    kfac.kfac_expert_forward(ctx, layer, None, offsets, x, W, want)
    wide = torch.full((E, 3, ci + 5), float("nan"), dtype=dtype, device="cuda")
    wide[:, 1:2, :ci] = W
    views = [wide[:, 1:2, :ci], W.transpose(1, 2).contiguous().transpose(1, 2), wide[:, 1:2]]
    for V in views:
        y = torch.empty_like(want)
        kfac.kfac_expert_forward(ctx, layer, None, offsets, x, V, y)
        torch.cuda.synchronize()
        assert torch.equal(y, want), V.stride()
    ctx.close()


def test_experts_that_lie_unevenly_are_refused():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    layer = wl.fc_layer(1, 8, 4, 0)
    ctx = kfac.Context([layer], workspace_bytes=256)
    W = torch.zeros(3, 6, 8, device="cuda")
    x, y, offsets = torch.zeros(5, 8, device="cuda"), torch.zeros(5, 4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (W[:, :4], W[:, :4].transpose(1, 2).contiguous().transpose(1, 2), W[:1, :4].expand(3, 4, 8)):
        with pytest.raises(ValueError):
            kfac.kfac_expert_forward(ctx, layer, None, offsets, x, bad, y)
    ctx.close()
