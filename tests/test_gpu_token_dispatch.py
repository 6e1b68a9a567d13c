"""Every kernel that the rules on sizes choose, on both sides of the rules, against the float64 definitions: those that the smaller
cases of the other files do not reach.  Tolerances as there: a sum of m terms within (m + 8) 2^-24 of the sum of their magnitudes (an
embedding's: m + 4), a bf16 result within 2^-8 of its value besides."""
import numpy as np
import pytest
import torch

from oracle import tokens as T
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


def _randn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def _check(got, ref, mag, m, what):
    bound = (m + 8) * 2.0 ** -24 * mag + (2.0 ** -8 * ref.abs() if got.dtype == BF16 else 0.0) + 1e-40
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bool(bad.any()), "%s: %d values" % (what, int(bad.sum()))


class Experts:
    """Choices with uneven experts, some of no expert, and the five products of a layer against float64."""

    def __init__(self, n, E, ci, co, bias, dtype):
        self.n, self.E, self.ci, self.co, self.bias, self.dtype = n, E, ci, co, bias, dtype
        rng = np.random.default_rng(n + E)
        p = 1.0 / np.arange(3, E + 4)
        self.choice = torch.from_numpy(rng.choice(np.concatenate([[-1], rng.permutation(E)]), n, p=p / p.sum()).astype(np.int32)).cuda()
        self.layer = wl.fc_layer(1, ci, co, bias)
        self.x, self.dy = _randn(1, n, ci).to(dtype), _randn(2, n, co).to(dtype)
        self.W = (_randn(3, E, co, ci + bias) / ci ** 0.5).to(dtype)
        self.order, self.offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
        self.ctx = kfac.Context([self.layer], workspace_bytes=max(kfac.kfac_segments_workspace_bytes(n, E), kfac.kfac_expert_workspace_bytes(self.layer, E, n)))
        kfac.kfac_segments(self.ctx, self.choice, E, self.order, self.offsets)

    def rows(self, e):
        mine = torch.nonzero(self.choice == e).reshape(-1)
        x, d, W = self.x[mine].double(), self.dy[mine].double(), self.W[e].double()
        return mine, torch.cat([x, torch.ones(mine.numel(), self.bias, dtype=torch.float64, device="cuda")], 1), d, W

    def products(self):
        y, dx = torch.full((self.n, self.co), 5.0, device="cuda").to(self.dtype), torch.full((self.n, self.ci), 5.0, device="cuda").to(self.dtype)
        kfac.kfac_expert_forward(self.ctx, self.layer, self.order, self.offsets, self.x, self.W, y)
        kfac.kfac_expert_grad_input(self.ctx, self.layer, self.order, self.offsets, self.dy, self.W, dx)
        free = self.choice < 0
        assert bool(free.any()) and not bool(y[free].any()) and not bool(dx[free].any())
        for e in range(self.E):
            mine, x, d, W = self.rows(e)
            _check(y[mine], x @ W.T, x.abs() @ W.abs().T, self.ci + 1, "y")
            W = W[:, :self.ci]
            _check(dx[mine], d @ W, d.abs() @ W.abs(), self.co, "dx")

    def contractions(self):
        E, ci, co, b = self.E, self.ci, self.co, self.bias
        dW, A, G = torch.full((E, co, ci + b), 5.0, device="cuda"), torch.full((E, ci + b, ci + b), 1.0, device="cuda"), torch.full((E, co, co), 1.0, device="cuda")
        kfac.kfac_expert_grad_weight(self.ctx, self.layer, self.order, self.offsets, self.x, self.dy, dW)
        kfac.kfac_stats_expert(self.ctx, self.layer, self.order, self.offsets, self.x, self.dy, 0.25, A, G)
        for e in range(E):
            mine, x, d, _ = self.rows(e)
            m = mine.numel()
            _check(dW[e], d.T @ x, d.abs().T @ x.abs(), m, "dW")
            for got, r, what in ((A[e], x, "A"), (G[e], d, "G")):
                old = 0.25 if m else 1.0
                _check(got, old + 0.75 * (r.T @ r) / max(1, m), old + 0.75 * (r.abs().T @ r.abs()) / max(1, m), m, what)
        assert torch.equal(A, A.transpose(1, 2)) and torch.equal(G, G.transpose(1, 2))


# bf16 in whole chunks: 64 x 64 below and 128 x 128 above 320 tiles of 128, 256 x 256 from 256 tiles of 256 on
@pytest.mark.parametrize("n,E,ci,co", [(2000, 16, 1024, 1024), (4100, 16, 1024, 1024), (4100, 16, 1032, 1096), (9000, 16, 1024, 1536)])
def test_bf16_tiles_straight_to_lds(n, E, ci, co):
    c = Experts(n, E, ci, co, 0, BF16)
    c.products()
    c.ctx.close()


@pytest.mark.parametrize("E,ci,co,bias", [(15, 1024, 1024, 0), (16, 1024, 1024, 1), (24, 520, 264, 1)])
def test_bf16_contractions_straight_to_lds(E, ci, co, bias):
    c = Experts(3000, E, ci, co, bias, BF16)
    c.contractions()
    c.ctx.close()


# any size: 64 x 64 with four and with two groups of waves, 128 x 128
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("fp32", [kfac.KFAC_PRODUCTS_SPLIT_BF16, kfac.KFAC_PRODUCTS_FP32_MFMA], ids=["planes", "fp32"])
@pytest.mark.parametrize("n,E,ci,co,bias", [(1500, 5, 131, 139, 1), (3000, 40, 131, 139, 1), (2500, 64, 101, 127, 1), (2500, 64, 127, 65, 0)])
def test_general_tiles(n, E, ci, co, bias, dtype, fp32):
    with kfac.default_options(fp32_products=fp32):
        c = Experts(n, E, ci, co, bias, dtype)
    c.products()
    c.contractions()
    c.ctx.close()


def test_rows_far_apart():
    """bf16 rows whose 32-bit offsets in bytes pass 2^31, and one row more, whose offsets pass 2^32: the general kernel takes these."""
    E, ci, co = 3, 64, 72
    ld = (1 << 31) // 300 // 8 * 8
    memory = torch.empty(301 * ld, dtype=BF16, device="cuda")
    for n in (300, 301):
        assert (n * ld < 1 << 31) == (n == 300)
        wide = memory[:n * ld].view(n, ld)
        c = Experts(n, E, ci, co, 0, BF16)
        x, dy = wide[:, 8:8 + ci], wide[:, 128:128 + co]
        x.copy_(c.x)
        dy.copy_(c.dy)
        c.x, c.dy = x, dy
        c.products()
        c.contractions()
        # results that lie as far apart
        y, z = wide[:, 256:256 + co], torch.empty(n, co, dtype=BF16, device="cuda")
        kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, x, c.W, y)
        kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, x, c.W, z)
        assert torch.equal(y, z)
        c.ctx.close()


def test_weights_far_apart():
    """The same of the rows of W: two experts of 2^32 bytes each."""
    n, E, ci, co = 200, 2, 72, 64
    for ldw in ((1 << 31) // co - 8, (1 << 31) // co + 8):
        c = Experts(n, E, ci, co, 0, BF16)
        W = torch.empty(E, co, ldw, dtype=BF16, device="cuda")[:, :, 16:16 + ci]
        W.copy_(c.W)
        c.W = W
        c.products()
        c.ctx.close()
        del W, c
        torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ segments, embedding
@pytest.mark.parametrize("n", [8192, 8193, 524288, 524289])
@pytest.mark.parametrize("num", [1, 31, 511, 512, 16383, 16384, 300000])
def test_segments_at_the_rules(n, num):
    """One workgroup and tiles (8192 positions), sums of the tiles in their own launch (524288), one pass of the sort and several
    (512 keys), offsets found by one workgroup and by several (16384 keys)."""
    ids = np.random.default_rng(n + num).integers(-1, num + 1, n)
    order, offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(num + 1, dtype=torch.int32, device="cuda")
    ctx = kfac.Context([wl.fc_layer(1, 4, 4)], workspace_bytes=kfac.kfac_segments_workspace_bytes(n, num))
    kfac.kfac_segments(ctx, torch.from_numpy(ids).cuda(), num, order, offsets)
    ref_order, ref_offsets = T.segments(ids, num)
    assert np.array_equal(order.cpu().numpy(), ref_order) and np.array_equal(offsets.cpu().numpy(), ref_offsets)
    ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,dim", [(32768, 256), (32769, 256), (16384, 1024), (16385, 1024), (32768, 1024), (32769, 1024), (70000, 1003)])
def test_embedding_gradient_at_the_rules(dtype, n, dim):
    """Runs of 8 positions and of 32 (32768 positions), gradients read through the caches and past them (64 MiB)."""
    vocab = 5000
    rng = np.random.default_rng(n + dim)
    p = 1.0 / np.arange(1, vocab + 1)
    ids = rng.choice(rng.permutation(vocab), n, p=p / p.sum())
    ids[rng.integers(0, n, n // 20)] = -1
    ids = torch.from_numpy(ids).cuda()
    g = _randn(n, n, dim + 1).to(dtype)[:, :dim]
    dW, A = torch.full((vocab, dim), float("nan"), device="cuda"), torch.full((vocab,), float("nan"), device="cuda")
    ctx = kfac.Context([wl.fc_layer(1, 4, 4)], workspace_bytes=kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
    kfac.kfac_embedding_grad(ctx, ids, g, 0.5, dW, False, A, 0.0)
    known = ids >= 0
    ref, mag = (torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, ids[known], v[known]) for v in (g.double(), g.double().abs()))
    counts = torch.bincount(ids[known], minlength=vocab)
    assert bool(((dW.double() - 0.5 * ref).abs() <= (counts[:, None] + 4) * 2.0 ** -24 * 0.5 * mag).all())
    assert torch.allclose(A.double(), counts.double() / n, rtol=8 * 2.0 ** -24, atol=0)
    ctx.close()
