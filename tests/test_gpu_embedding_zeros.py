"""Rows of tokens that do not occur become zero in tables of any size, the smallest ones too."""
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


@pytest.mark.parametrize("n", [0, 1, 5, 8192, 9000])
@pytest.mark.parametrize("with_diagonal", [False, True])
def test_gradient_of_small_tables(n, with_diagonal):
    """Every table of up to 40 elements, with no token, and with token 0 alone."""
    for size in range(1, 41):
        for dim in (d for d in range(1, size + 1) if size % d == 0):
            vocab = size // dim
            ctx = kfac.Context([wl.fc_layer(1, 4, 4)], workspace_bytes=kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
            grad = torch.ones(n, dim, device="cuda")
            for token in (-1, 0):
                ids = torch.full((n,), token, dtype=torch.int64, device="cuda")
                buf = torch.full((size + 4,), float("nan"), device="cuda")
                A = torch.full((vocab,), float("nan"), device="cuda") if with_diagonal else None
                kfac.kfac_embedding_grad(ctx, ids, grad, 1.0, buf[:size].view(vocab, dim), False, A, 0.0)
                want = torch.zeros(size, device="cuda")
                if token == 0:
                    want[:dim] = float(n)                  # n ones: exact
                assert torch.equal(buf[:size], want), (vocab, dim, token)
                assert bool(torch.isnan(buf[size:]).all()), (vocab, dim, token)
                if with_diagonal and n > 0:
                    assert abs(float(A[0]) - (token == 0)) <= 2.0 ** -22 and not bool(A[1:].any()), (vocab, dim, token)
            ctx.close()
