"""Inputs and outputs that are columns of one wider tensor, beside each other: they do not overlap."""
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


def _wide(rows, cols, dtype, seed=1):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(rows, cols, generator=g).cuda().to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first", [False, True])
def test_dropout_and_lookup(dtype, first):
    """x and y (table and out) as the two halves of the columns, in either order, a residual between them."""
    rows, d = 37, 40
    t = _wide(rows, 3 * d, dtype)
    before = t.clone()
    x, r, y = (t[:, i * d:(i + 1) * d] for i in ((0, 1, 2) if first else (2, 1, 0)))
    ctx = kfac.Context([wl.fc_layer(1, 4, 4)], workspace_bytes=256)
    want = torch.empty(rows, d, dtype=dtype, device="cuda")
    kfac.kfac_dropout(ctx, x.contiguous(), 0.3, 5, 6, want, residual=r.contiguous())
    kfac.kfac_dropout(ctx, x, 0.3, 5, 6, y, residual=r)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(t[:, d:2 * d], before[:, d:2 * d])
    assert torch.equal(x, before[:, :d] if first else before[:, 2 * d:])
    ids = (torch.arange(rows, dtype=torch.int32) * 7 % rows).cuda()
    kfac.kfac_embedding(ctx, ids, x, 1.0, y)
    torch.cuda.synchronize()
    assert torch.equal(y, x[ids.long()])
    ctx.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ci,co", [(64, 32), (61, 33)])
def test_experts(dtype, ci, co):
    n, E = 50, 3
    layer = wl.fc_layer(1, ci, co, 0)
    t = _wide(n, 2 * (ci + co), dtype)
    W = _wide(E * co, ci, dtype, 2).view(E, co, ci)
    x, y, dy, dx = t[:, :ci], t[:, ci:ci + co], t[:, ci + co:ci + 2 * co], t[:, ci + 2 * co:]
    offsets = torch.tensor([0, 20, 20, n], dtype=torch.int32).cuda()
    ctx = kfac.Context([layer], workspace_bytes=kfac.kfac_expert_workspace_bytes(layer, E, n))
    want_y, want_dx = torch.empty(n, co, dtype=dtype, device="cuda"), torch.empty(n, ci, dtype=dtype, device="cuda")
    kfac.kfac_expert_forward(ctx, layer, None, offsets, x.contiguous(), W, want_y)
    kfac.kfac_expert_grad_input(ctx, layer, None, offsets, dy.contiguous(), W, want_dx)
    before = t.clone()
    kfac.kfac_expert_forward(ctx, layer, None, offsets, x, W, y)
    kfac.kfac_expert_grad_input(ctx, layer, None, offsets, dy, W, dx)
    torch.cuda.synchronize()
    assert torch.equal(y, want_y) and torch.equal(dx, want_dx)
    assert torch.equal(x, before[:, :ci]) and torch.equal(dy, before[:, ci + co:ci + 2 * co])
    ctx.close()
