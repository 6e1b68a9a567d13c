"""Products grouped by expert, their gradients and factors on the GPU against their float64 definitions.

Tolerances: a sum of m products formed in fp32 is within (m + 8) 2^-24 of the sum of their magnitudes (the terms that three bf16
planes leave out are below 3 * 2^-24 of a product), a bf16 output within 2^-8 of its value besides."""
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


def _layer(ci, co, bias):
    return wl.fc_layer(1, ci, co, bias)


def _choices(rng, n, E, kind):
    if kind == "skew":
        p = 1.0 / np.arange(1, E + 1) ** 1.5
        c = rng.choice(E, n, p=p / p.sum())
    elif kind == "one":
        c = np.full(n, E - 1)
    elif kind == "none":
        c = np.full(n, -1)
    elif kind == "drop":
        c = rng.integers(-1, E + 1, n)
    else:
        c = rng.integers(0, E, n)
    if kind == "skew" and E > 2:
        c[c == 1] = 0                                               # an expert without rows
    return c.astype(np.int32)


def _rows(a, dtype, pad=0, fill=float("nan")):
    t = torch.full((a.shape[0], a.shape[1] + pad), fill, dtype=dtype, device="cuda")
    t[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t[:, :a.shape[1]]


def _values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _close(got, ref, mag, m, dtype, what):
    bound = (m + 8) * 2.0 ** -24 * mag + (2.0 ** -8 * np.abs(ref) if dtype == BF16 else 0.0) + 1e-40
    bad = ~(np.abs(_values(got) - ref) <= bound)
    assert not bad.any(), "%s: %d of %d, worst %.3g of its bound" % (what, bad.sum(), bad.size, np.nanmax(np.abs(_values(got) - ref) / bound))


class Case:
    def __init__(self, tokens, fan, E, ci, co, bias, dtype, kind, pad=0, seed=0):
        rng = np.random.default_rng(seed + tokens + 7 * ci + co)
        self.tokens, self.fan, self.E, self.ci, self.co, self.bias, self.dtype = tokens, fan, E, ci, co, bias, dtype
        self.n = n = tokens * fan
        self.layer = _layer(ci, co, bias)
        self.choice = _choices(rng, n, E, kind)
        self.x, self.dy = _rows(rng.standard_normal((tokens, ci)), dtype, pad), _rows(rng.standard_normal((n, co)), dtype, pad)
        W = torch.full((E, co, ci + bias + pad), float("nan"), dtype=dtype, device="cuda")
        W[:, :, :ci + bias] = torch.from_numpy(rng.standard_normal((E, co, ci + bias)) / np.sqrt(ci)).to(dtype)
        self.W = W
        self.order, self.offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
        self.ctx = kfac.Context([self.layer], workspace_bytes=max(kfac.kfac_segments_workspace_bytes(n, E), kfac.kfac_expert_workspace_bytes(self.layer, E, n)))
        kfac.kfac_segments(self.ctx, torch.from_numpy(self.choice).cuda(), E, self.order, self.offsets)
        self.longest = int(np.bincount(self.choice[(self.choice >= 0) & (self.choice < E)], minlength=1).max()) if n else 0

    def out(self, cols, pad):
        self.whole = torch.full((self.n + 1, cols + pad), 5.0, dtype=self.dtype, device="cuda")
        return self.whole[:self.n, :cols]

    def untouched(self, cols):
        return bool((self.whole[self.n] == 5.0).all()) and bool((self.whole[:, cols:] == 5.0).all())


SHAPES = [  # tokens, fan, experts, c_in, c_out, bias, kind, pad
    (1, 1, 1, 1, 1, 0, "even", 0),
    (1, 2, 4, 64, 64, 0, "even", 0),
    (3, 2, 16, 128, 72, 0, "even", 0),
    (5, 1, 3, 7, 9, 1, "even", 3),
    (33, 1, 4, 515, 33, 1, "skew", 0),
    (64, 4, 8, 256, 128, 0, "skew", 8),
    (130, 2, 5, 100, 257, 1, "drop", 0),
    (200, 1, 70, 64, 136, 0, "even", 0),
    (300, 1, 2, 384, 512, 0, "one", 0),
    (90, 1, 3, 40, 48, 1, "none", 0),
    (1031, 2, 6, 192, 320, 0, "skew", 0),
    (700, 1, 4, 264, 520, 1, "drop", 8),
]
IDS = ["x".join(str(v) for v in s) for s in SHAPES]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward_and_gradients(shape, dtype):
    tokens, fan, E, ci, co, bias, kind, pad = shape
    c = Case(tokens, fan, E, ci, co, bias, dtype, kind, pad)
    x, dy, W = _values(c.x), _values(c.dy), _values(c.W)
    y = c.out(co, pad)
    kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, c.x, c.W, y, fan=fan)
    torch.cuda.synchronize()
    ref, mag = T.expert_forward(c.choice, x, W, ci, bias, fan)
    _close(y, ref, mag, ci + 1, dtype, "y")
    assert c.untouched(co)
    dx = c.out(ci, pad)
    kfac.kfac_expert_grad_input(c.ctx, c.layer, c.order, c.offsets, c.dy, c.W, dx)
    torch.cuda.synchronize()
    ref, mag = T.expert_grad_input(c.choice, dy, W, ci)
    _close(dx, ref, mag, co, dtype, "dx")
    assert c.untouched(ci)
    buf = torch.full((E * co * (ci + bias) + 8,), 5.0, device="cuda")
    dW = buf[:-8].view(E, co, ci + bias)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW, fan=fan)
    torch.cuda.synchronize()
    ref, mag = T.expert_grad_weight(c.choice, x, dy, E, bias, fan)
    _close(dW, ref, mag, c.longest, F32, "dW")
    assert bool((buf[-8:] == 5.0).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_factors(shape, dtype):
    tokens, fan, E, ci, co, bias, kind, pad = shape
    c = Case(tokens, fan, E, ci, co, bias, dtype, kind, pad, seed=5)
    x, dy = _values(c.x), _values(c.dy)
    rng = np.random.default_rng(4)
    for decay in (0.0, 0.95):
        A0, G0 = rng.standard_normal((E, ci + bias, ci + bias)).astype(np.float32), rng.standard_normal((E, co, co)).astype(np.float32)
        A0, G0 = A0 + A0.transpose(0, 2, 1), G0 + G0.transpose(0, 2, 1)
        refA, magA, count = T.expert_factors(c.choice, x, E, bias, fan)
        refG, magG, _ = T.expert_factors(c.choice, dy, E, 0, 1)
        empty = count == 0
        if decay == 0.0:
            A0[~empty], G0[~empty] = np.nan, np.nan                 # never read
        A, G = torch.from_numpy(A0).cuda(), torch.from_numpy(G0).cuda()
        kfac.kfac_stats_expert(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, decay, A, G, fan=fan)
        torch.cuda.synchronize()
        d = np.float64(np.float32(decay))
        for got, old, ref, mag, what in ((A, A0, refA, magA, "A"), (G, G0, refG, magG, "G")):
            g = got.cpu().numpy()
            assert np.array_equal(g[empty], old[empty]), what       # an expert without rows keeps its factors
            if (~empty).any():
                old = old[~empty].astype(np.float64) if decay else 0.0
                _close(got[torch.from_numpy(~empty).cuda()], d * old + (1 - d) * ref[~empty], d * np.abs(old) + (1 - d) * mag[~empty], c.longest, F32, what)
                assert np.array_equal(g[~empty], g[~empty].transpose(0, 2, 1))
        # one factor alone
        B = torch.from_numpy(A0).cuda()
        kfac.kfac_stats_expert(c.ctx, c.layer, c.order, c.offsets, c.x, None, decay, B, None, fan=fan)
        H = torch.from_numpy(G0).cuda()
        kfac.kfac_stats_expert(c.ctx, c.layer, c.order, c.offsets, None, c.dy, decay, None, H, fan=fan)
        torch.cuda.synchronize()
        assert torch.equal(B.view(torch.int32), A.view(torch.int32)) and torch.equal(H.view(torch.int32), G.view(torch.int32))
    c.ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ci,co,bias", [(64, 96, 0), (61, 33, 1)])
def test_nan_stays_where_it_is(dtype, ci, co, bias):
    """A NaN in a row reaches the row's own outputs and its expert's sums, nothing else; one in a row that no expert takes nothing."""
    c = Case(150, 1, 4, ci, co, bias, dtype, "drop")
    ctx = c.ctx
    clean = [c.out(co, 0), torch.empty(4, co, ci + bias, device="cuda"), torch.empty(4, ci + bias, ci + bias, device="cuda"), torch.empty(4, co, co, device="cuda")]
    kfac.kfac_expert_forward(ctx, c.layer, c.order, c.offsets, c.x, c.W, clean[0])
    kfac.kfac_expert_grad_weight(ctx, c.layer, c.order, c.offsets, c.x, c.dy, clean[1])
    kfac.kfac_stats_expert(ctx, c.layer, c.order, c.offsets, c.x, c.dy, 0.0, clean[2], clean[3])
    victim = int(np.nonzero(c.choice == 2)[0][3])
    nobody = np.nonzero((c.choice < 0) | (c.choice >= 4))[0]
    c.x[victim], c.dy[victim] = float("nan"), float("inf")
    c.x[torch.from_numpy(nobody).cuda()] = float("nan")
    c.dy[torch.from_numpy(nobody).cuda()] = float("nan")
    y = torch.empty_like(clean[0])
    got = [y, torch.empty_like(clean[1]), torch.empty_like(clean[2]), torch.empty_like(clean[3])]
    kfac.kfac_expert_forward(ctx, c.layer, c.order, c.offsets, c.x, c.W, y)
    kfac.kfac_expert_grad_weight(ctx, c.layer, c.order, c.offsets, c.x, c.dy, got[1])
    kfac.kfac_stats_expert(ctx, c.layer, c.order, c.offsets, c.x, c.dy, 0.0, got[2], got[3])
    torch.cuda.synchronize()
    rows = torch.ones(150, dtype=torch.bool, device="cuda")
    rows[victim] = False
    assert torch.equal(y[rows], clean[0][rows]) and bool(torch.isnan(y[victim]).all())
    for g, ref in zip(got[1:], clean[1:]):
        others = [e for e in range(4) if e != 2]
        assert torch.equal(g[others], ref[others]) and not bool(torch.isfinite(g[2]).all())
    ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sorted_choices_need_no_order(dtype):
    c = Case(260, 1, 3, 128, 64, 0, dtype, "even")
    back = c.order.long()
    xs, dys = c.x[back].contiguous(), c.dy[back].contiguous()
    y, dx, dW = c.out(64, 0).clone(), torch.empty(260, 128, dtype=dtype, device="cuda"), torch.empty(3, 64, 128, device="cuda")
    y2, dx2, dW2 = torch.empty_like(y), torch.empty_like(dx), torch.empty_like(dW)
    kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, c.x, c.W, y)
    kfac.kfac_expert_grad_input(c.ctx, c.layer, c.order, c.offsets, c.dy, c.W, dx)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW)
    kfac.kfac_expert_forward(c.ctx, c.layer, None, c.offsets, xs, c.W, y2)
    kfac.kfac_expert_grad_input(c.ctx, c.layer, None, c.offsets, dys, c.W, dx2)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, None, c.offsets, xs, dys, dW2)
    torch.cuda.synchronize()
    assert torch.equal(y[back], y2) and torch.equal(dx[back], dx2) and torch.equal(dW, dW2)
    c.ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_offsets_out_of_range_stay_inside_the_tensors(dtype):
    """Offsets and places that no call of kfac_segments makes: read as empty or cut off, nothing behind the tensors is touched."""
    n, ci, co = 40, 64, 64
    c = Case(n, 1, 3, ci, co, 0, dtype, "even")
    order = c.order.clone()
    order[5], order[7] = -3, n + 9
    offsets = torch.tensor([-5, 30, 10, n + 100], dtype=torch.int32, device="cuda")
    y = c.out(co, 0)
    dW, A = torch.empty(3, co, ci, device="cuda"), torch.zeros(3, ci, ci, device="cuda")
    kfac.kfac_expert_forward(c.ctx, c.layer, order, offsets, c.x, c.W, y)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, order, offsets, c.x, c.dy, dW)
    kfac.kfac_stats_expert(c.ctx, c.layer, order, offsets, c.x, None, 0.0, A, None)
    torch.cuda.synchronize()
    assert c.untouched(co) and bool(torch.isfinite(dW).all()) and bool(torch.isfinite(A).all())
    c.ctx.close()


def test_gradients_by_differences():
    """The loss sum(y * R) is linear in x and in W: difference quotients of the forward product are its gradients."""
    c = Case(40, 2, 3, 24, 20, 1, F32, "drop")
    R = c.dy
    y, dx, dW = torch.empty(80, 20, device="cuda"), torch.empty(80, 24, device="cuda"), torch.empty(3, 20, 25, device="cuda")
    kfac.kfac_expert_grad_input(c.ctx, c.layer, c.order, c.offsets, R, c.W, dx)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, R, dW, fan=2)
    dx = dx.view(40, 2, 24).sum(1)

    def loss(x, W):
        kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, x, W, y, fan=2)
        return float((y.double() * R.double()).sum())

    # h = 1: 1600 outputs of a few units, each within (25 + 8) 2^-24 of the sum of its magnitudes (below 32), times |R| below 5
    tol = 1600 * 33 * 2.0 ** -24 * 32 * 5 / 100
    for t, k in ((0, 0), (7, 11), (39, 23)):
        step = torch.zeros_like(c.x)
        step[t, k] = 1.0
        assert abs((loss(c.x + step, c.W) - loss(c.x - step, c.W)) / 2 - float(dx[t, k])) < tol
    for e, o, k in ((0, 0, 0), (1, 13, 7), (2, 19, 24)):
        step = torch.zeros_like(c.W)
        step[e, o, k] = 1.0
        assert abs((loss(c.x, c.W + step) - loss(c.x, c.W - step)) / 2 - float(dW[e, o, k])) < tol
    c.ctx.close()


def test_no_choices():
    layer = _layer(16, 8, 1)
    ctx = kfac.Context([layer], workspace_bytes=kfac.kfac_expert_workspace_bytes(layer, 4, 0))
    offsets = torch.zeros(5, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, 16, device="cuda")
    y = torch.empty(0, 8, device="cuda")
    dW, A = torch.full((4, 8, 17), 3.0, device="cuda"), torch.full((4, 17, 17), 3.0, device="cuda")
    W = torch.randn(4, 8, 17, device="cuda")
    kfac.kfac_expert_forward(ctx, layer, None, offsets, empty, W, y)
    kfac.kfac_expert_grad_input(ctx, layer, None, offsets, y, W, empty)
    kfac.kfac_expert_grad_weight(ctx, layer, None, offsets, empty, y, dW)
    kfac.kfac_stats_expert(ctx, layer, None, offsets, empty, None, 0.5, A, None)
    torch.cuda.synchronize()
    assert not bool(dW.any()) and bool((A == 3.0).all())
    ctx.close()


def test_experts_under_the_natural_gradient():
    """Factors of experts go through kfac_invert and kfac_precondition as those of any fully-connected layer."""
    import oracle
    c = Case(300, 1, 3, 32, 16, 1, F32, "even")
    E, dA, dG = 3, 33, 16
    A, G = torch.zeros(E, dA, dA, device="cuda"), torch.zeros(E, dG, dG, device="cuda")
    dW = torch.empty(E, dG, dA, device="cuda")
    layers = [c.layer] * E
    ctx = kfac.Context(layers)
    kfac.kfac_stats_expert(ctx, c.layer, c.order, c.offsets, c.x, c.dy, 0.0, A, G)
    kfac.kfac_expert_grad_weight(ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW)
    Ai, Gi, U = torch.empty_like(A), torch.empty_like(G), torch.empty_like(dW)
    info = torch.zeros(2 * E, dtype=torch.int32, device="cuda")
    kfac.kfac_invert(ctx, layers, list(A), list(G), 0.05, list(Ai), list(Gi), None, info)
    kfac.kfac_precondition(ctx, layers, list(Gi), list(Ai), list(dW), list(U))
    torch.cuda.synchronize()
    assert not bool(info.any())
    refA, _, _ = T.expert_factors(c.choice, _values(c.x), E, 1, 1)
    refG, _, _ = T.expert_factors(c.choice, _values(c.dy), E, 0, 1)
    refW, _ = T.expert_grad_weight(c.choice, _values(c.x), _values(c.dy), E, 1, 1)
    for e in range(E):
        Ari, Gri, _, _ = oracle.kfac_invert(refA[e], refG[e], 0.05)
        ref = oracle.kfac_precondition(Gri, Ari, refW[e])
        # the bar of the preconditioned gradient in the parity tests
        assert np.abs(_values(U[e]) - ref).max() <= 1e-3 * np.abs(ref).max()
    ctx.close()
    c.ctx.close()


@pytest.mark.parametrize("ci,co,bias,dtype", [(1032, 1032, 0, BF16), (1032, 1040, 1, BF16), (1033, 1030, 0, BF16), (1033, 1030, 1, F32)])
def test_many_tiles(ci, co, bias, dtype):
    """Enough rows and columns for the largest tiles; ragged segments, choices that no expert takes, gathered rows two to a token."""
    tokens, fan, E = 5000, 2, 16
    c = Case(tokens, fan, E, ci, co, bias, dtype, "drop", 0, seed=2)
    n = c.n
    choice = torch.from_numpy(c.choice).cuda()
    y, dx, dW = c.out(co, 0), torch.full((n, ci), 5.0, dtype=dtype, device="cuda"), torch.full((E, co, ci + bias), 5.0, device="cuda")
    A, G = torch.full((E, ci + bias, ci + bias), 1.0, device="cuda"), torch.full((E, co, co), 1.0, device="cuda")
    kfac.kfac_expert_forward(c.ctx, c.layer, c.order, c.offsets, c.x, c.W, y, fan=fan)
    kfac.kfac_expert_grad_input(c.ctx, c.layer, c.order, c.offsets, c.dy, c.W, dx)
    kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW, fan=fan)
    kfac.kfac_stats_expert(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, 0.5, A, G, fan=fan)
    torch.cuda.synchronize()
    assert c.untouched(co)

    def check(got, ref, mag, m, out, what):
        bound = (m + 8) * 2.0 ** -24 * mag + (2.0 ** -8 * ref.abs() if out == BF16 else 0.0) + 1e-40
        bad = ~((got.double() - ref).abs() <= bound)
        assert not bool(bad.any()), "%s: %d values" % (what, int(bad.sum()))

    free = (choice < 0) | (choice >= E)
    assert not bool(y[free].any()) and not bool(dx[free].any()) and bool(free.any())
    for e in range(E):
        mine = torch.nonzero(choice == e).reshape(-1)
        m = mine.numel()
        x, d, W = c.x[mine // fan].double(), c.dy[mine].double(), c.W[e, :, :ci].double()
        b = c.W[e, :, ci].double() if bias else torch.zeros(co, dtype=torch.float64, device="cuda")
        check(y[mine], x @ W.T + b, x.abs() @ W.abs().T + b.abs(), ci + 1, dtype, "y")
        check(dx[mine], d @ W, d.abs() @ W.abs(), co, dtype, "dx")
        if bias:
            x = torch.cat([x, torch.ones(m, 1, dtype=torch.float64, device="cuda")], 1)
        check(dW[e], d.T @ x, d.abs().T @ x.abs(), m, F32, "dW")
        check(A[e], 0.5 + 0.5 * (x.T @ x) / m, 0.5 + 0.5 * (x.abs().T @ x.abs()) / m, m, F32, "A")
        check(G[e], 0.5 + 0.5 * (d.T @ d) / m, 0.5 + 0.5 * (d.abs().T @ d.abs()) / m, m, F32, "G")
    assert torch.equal(A, A.transpose(1, 2)) and torch.equal(G, G.transpose(1, 2))
    c.ctx.close()


def test_rows_of_all_lengths_of_a_contraction():
    """Weight gradients over segments of 0 .. 200 rows: every length of the last, partial step, whole steps and none."""
    E, ci, co = 201, 72, 40
    lengths = np.arange(E)
    np.random.default_rng(0).shuffle(lengths)
    choice = np.repeat(np.arange(E), lengths).astype(np.int32)
    n = len(choice)
    for dtype in (F32, BF16):
        c = Case(n, 1, E, ci, co, 0, dtype, "even")
        kfac.kfac_segments(c.ctx, torch.from_numpy(choice).cuda(), E, c.order, c.offsets)
        dW = torch.full((E, co, ci), 5.0, device="cuda")
        kfac.kfac_expert_grad_weight(c.ctx, c.layer, c.order, c.offsets, c.x, c.dy, dW)
        ref, mag = T.expert_grad_weight(choice, _values(c.x), _values(c.dy), E, 0, 1)
        _close(dW, ref, mag, 200, F32, "dW")
        c.ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_captured_in_a_graph(dtype):
    """The calls in a HIP graph, replayed with other inputs and with eager work between the replays."""
    stream = torch.cuda.Stream()
    layer = _layer(128, 64, 0)
    n, E = 300, 4
    with torch.cuda.stream(stream):
        ctx = kfac.Context([layer], workspace_bytes=max(kfac.kfac_segments_workspace_bytes(n, E), kfac.kfac_embedding_workspace_bytes(n, 50, 128)), stream=stream)
        choice = torch.zeros(n, dtype=torch.int32, device="cuda")
        x, W, dy = (torch.randn(*s, device="cuda").to(dtype) for s in ((n, 128), (E, 64, 128), (n, 64)))
        order, offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
        y, dW, dT = torch.empty(n, 64, dtype=dtype, device="cuda"), torch.empty(E, 64, 128, device="cuda"), torch.empty(50, 128, device="cuda")
        h = torch.empty_like(x)

        def run():
            kfac.kfac_segments(ctx, choice, E, order, offsets)
            kfac.kfac_dropout(ctx, x, 0.3, 5, 6, h)
            kfac.kfac_expert_forward(ctx, layer, order, offsets, h, W, y)
            kfac.kfac_expert_grad_weight(ctx, layer, order, offsets, h, dy, dW)
            kfac.kfac_embedding_grad(ctx, choice, h, 1.0, dT)

        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for k in range(4):
            choice.copy_(torch.randint(-1, E, (n,), device="cuda"))
            x.copy_(torch.randn(n, 128, device="cuda"))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in (order, offsets, y, dW, dT)]
            run()
            stream.synchronize()
            for a, b in zip(got, (order, offsets, y, dW, dT)):
                assert torch.equal(a, b)
        ctx.close()
