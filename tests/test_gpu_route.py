"""Routing and its gradient on the GPU against their float64 definitions.

Tolerances, in units of 2^-24 of the value: expf and its argument 4 + the largest difference of two logits that count (its
rounding), a sum of m positive terms m, quotients and products 8; gradients: the same of the magnitudes that are added up.  An output in
bf16 is within 2^-8 of its value besides.  Choices are exact."""
import numpy as np
import pytest
import torch

from oracle import blocks as B
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    c = kfac.Context([wl.fc_layer(2, 64, 32)], workspace_bytes=256)
    yield c
    c.close()


def _rows(a, dtype, pad=0, fill=float("nan")):
    t = torch.full((a.shape[0] + 1, a.shape[1] + pad), fill, dtype=dtype, device="cuda")
    t[:-1, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t[:-1, :a.shape[1]], t


def _values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _run(ctx, logits, bias, d, dtype, pad, **options):
    """Forward and gradient against the oracle; logits, bias, d: numpy."""
    n, E = logits.shape
    r = kfac.router(E, **{k: (int(v) if k == "scores" else v) for k, v in options.items()})
    fan, sigmoid = r.fan, r.scores == kfac.KFAC_ROUTE_SIGMOID
    x, _ = _rows(logits, dtype, pad)
    b = None if bias is None else torch.from_numpy(bias.astype(np.float32)).cuda()
    choice, gate = torch.full((n * fan + 3,), -7, dtype=torch.int32, device="cuda"), torch.full((n * fan + 3,), 5.0, device="cuda")
    kfac.kfac_route(ctx, r, x, choice[:n * fan], gate[:n * fan], bias=b)
    torch.cuda.synchronize()
    l = _values(x)
    more = dict(sigmoid=sigmoid, renormalise=bool(r.renormalise), scale=float(r.scale))
    ref, refg = B.route(l, None if b is None else b.cpu().double().numpy(), fan, r.groups, r.top_groups, r.group_best, **more)
    got = choice.cpu().numpy()
    assert np.array_equal(got[:n * fan].reshape(n, fan), ref) and (got[n * fan:] == -7).all()
    g = gate.cpu().double().numpy()
    assert (g[n * fan:] == 5.0).all()
    g = g[:n * fan].reshape(n, fan)
    fine = np.where(np.isfinite(l), l, np.nan)
    spread = np.nan_to_num(np.nanmax(fine, 1, initial=-1e30) - np.nanmin(fine, 1, initial=1e30)).clip(0)[:, None] if E else 0
    units = 2 * spread + 40 + E + fan
    assert np.array_equal(np.isnan(g), np.isnan(refg))
    ok = ~np.isnan(refg)
    assert (np.abs(g - refg)[ok] <= (units * 2.0 ** -24 * np.abs(refg) + 1e-37)[ok]).all()

    up = torch.from_numpy(d.astype(np.float32)).cuda()
    out, whole = _rows(np.zeros((n, E)), dtype, pad, 5.0)
    kfac.kfac_route_grad(ctx, r, x, choice[:n * fan], up, out)
    torch.cuda.synchronize()
    refd, mag = B.route_grad(l, ref, up.cpu().double().numpy().reshape(n, fan), **more)
    assert (np.abs(_values(out) - refd) <= units * 2.0 ** -24 * mag + (UNIT[dtype] * np.abs(refd)) + 1e-37).all()
    assert bool((whole[-1] == 5.0).all()) and bool((whole[:, E:] == 5.0).all())
    return ref


CASES = [  # n, experts, options, pad
    (0, 8, dict(fan=2), 0),
    (1, 1, dict(fan=1), 0),
    (1, 8, dict(fan=8), 0),
    (3, 5, dict(fan=2), 3),
    (4, 64, dict(fan=2), 0),
    (5, 1024, dict(fan=32), 0),
    (63, 7, dict(fan=3, renormalise=False), 1),
    (65, 16, dict(fan=4, scale=-2.5), 0),
    (70, 17, dict(fan=4), 5),
    (33, 60, dict(fan=6, groups=4, top_groups=2), 0),
    (40, 64, dict(fan=8, groups=8, top_groups=3, group_best=2), 0),
    (40, 64, dict(fan=4, groups=64, top_groups=7), 2),
    (50, 128, dict(fan=8), 0),
    (30, 160, dict(fan=6, groups=8, top_groups=3, group_best=2, scale=16.0), 8),
    (64, 256, dict(fan=8, groups=8, top_groups=4, group_best=2, scale=2.5), 0),
    (21, 384, dict(fan=8, renormalise=False), 0),
    (19, 500, dict(fan=1, groups=2, top_groups=1, renormalise=False), 0),
    (9, 1024, dict(fan=16, groups=256, top_groups=5, group_best=2), 0),
    (7, 1000, dict(fan=31, groups=125, top_groups=125), 0),
    (1029, 32, dict(fan=2), 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scores", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True], ids=["", "bias"])
@pytest.mark.parametrize("case", CASES, ids=["%dx%d_%d" % (c[0], c[1], i) for i, c in enumerate(CASES)])
def test_route(ctx, case, with_bias, scores, dtype):
    n, E, options, pad = case
    rng = np.random.default_rng(n + E + scores)
    logits = rng.standard_normal((n, E)) * 2
    logits[rng.random((n, E)) < 0.05] = -INF                        # closed experts
    if n > 8:
        logits[3] = -INF                                            # padding
        logits[4, 1:] = -INF                                        # one expert left
        logits[5] = 0.25                                            # all alike
    bias = 0.1 * rng.standard_normal(E) if with_bias else None
    _run(ctx, logits, bias, rng.standard_normal((n, options["fan"])), dtype, pad, scores=scores, **options)


@pytest.mark.parametrize("scores", [0, 1])
@pytest.mark.parametrize("bias", ["zero", "steps", "huge", "near"])
def test_equal_and_nearly_equal_ranks(ctx, bias, scores):
    """Logits of few values, so that most ranks have an equal or a nearly equal neighbour; biases that are all alike, of few values, so
    large that fp32 would swallow the scores, and differences of logits that a bias nearly takes back."""
    rng = np.random.default_rng(7)
    n, E = 200, 64
    logits = rng.integers(-3, 4, (n, E)) / 4.0
    b = {"zero": np.zeros(E), "steps": rng.integers(0, 3, E) * 1e-3, "huge": np.full(E, 2.0 ** 20), "near": np.zeros(E)}[bias]
    if bias == "near":                                              # ranks of pairs that differ by less than fp32 resolves
        logits = np.repeat(rng.standard_normal((n, E // 2)), 2, 1).astype(np.float32)
        logits[:, 1::2] = np.nextafter(logits[:, 1::2], np.float32(9), dtype=np.float32)
    for groups, top, best in ((1, 1, 1), (8, 4, 2)):
        _run(ctx, logits, b, rng.standard_normal((n, 6)), F32, 0, scores=scores, fan=6, groups=groups, top_groups=top, group_best=best)
        _run(ctx, logits, None, rng.standard_normal((n, 6)), F32, 0, scores=scores, fan=6, groups=groups, top_groups=top, group_best=best)


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("scores", [0, 1])
def test_values_at_the_ends(ctx, scores, renormalise):
    rng = np.random.default_rng(8)
    logits = rng.standard_normal((40, 24))
    logits[0] = -np.arange(24) * 5.0 - 70                           # sigmoids beyond the range of fp32
    logits[1] = np.arange(24) * 4.0                                 # sigmoids of one, softmaxes of nearly zero
    logits[2] = -3e38
    logits[3, 7] = np.nan
    logits[4, 7] = INF
    logits[5] = INF
    logits[6, :20] = -INF
    logits[7] = 3e38
    d = rng.standard_normal((40, 6))
    if scores == 1 and not renormalise:
        logits[0] = -np.arange(24) - 40                             # (values in fp32's range)
    _run(ctx, logits, None, d, F32, 0, scores=scores, fan=6, renormalise=renormalise)
    bias = rng.standard_normal(24)
    bias[3], bias[5], bias[9] = -INF, INF, -INF
    choice = _run(ctx, logits, bias, d, F32, 0, scores=scores, fan=6, renormalise=renormalise)
    assert not np.isin(choice, (3, 9)).any()
    bias[4] = np.nan
    assert (_run(ctx, logits, bias, d, F32, 0, scores=scores, fan=6, renormalise=renormalise)[8:] == -1).all()


def test_gradient_of_any_choices(ctx):
    """The same expert twice, choices outside the range with NaN beside them, in any order."""
    rng = np.random.default_rng(9)
    l, d = rng.standard_normal((50, 12)), rng.standard_normal((50, 5)).astype(np.float32)
    c = rng.integers(-2, 14, (50, 5))
    c[0] = 3
    c[1] = -1
    c[2] = [1, 1, 2, 2, 100]
    d[(c < 0) | (c >= 12)] = np.nan
    x, _ = _rows(l, F32)
    for scores in (0, 1):
        for renormalise in (False, True):
            r = kfac.router(12, 5, scores=scores, renormalise=renormalise, scale=1.5)
            out, _ = _rows(np.zeros((50, 12)), F32)
            kfac.kfac_route_grad(ctx, r, x, torch.from_numpy(c.reshape(-1).astype(np.int32)).cuda(), torch.from_numpy(d).cuda(), out)
            ref, mag = B.route_grad(_values(x), c, d.astype(np.float64), sigmoid=scores == 1, renormalise=renormalise, scale=1.5)
            assert (np.abs(_values(out) - ref) <= 80 * 2.0 ** -24 * mag + 2.0 ** -24 * np.abs(ref)).all()


def test_routing_sorts_into_segments(ctx):
    """Choices of -1 and tokens with NaN go behind the last segment, and their rows of the product are zero."""
    rng = np.random.default_rng(10)
    l = rng.standard_normal((100, 6))
    l[10], l[20, 3] = -INF, np.nan
    x, _ = _rows(l, F32)
    r = kfac.router(6, 2)
    choice, gate = torch.empty(200, dtype=torch.int32, device="cuda"), torch.empty(100, 2, device="cuda")
    kfac.kfac_route(ctx, r, x, choice, gate)
    c = kfac.Context([wl.fc_layer(2, 8, 4)], workspace_bytes=kfac.kfac_segments_workspace_bytes(200, 6))
    order, offsets = torch.empty(200, dtype=torch.int32, device="cuda"), torch.empty(7, dtype=torch.int32, device="cuda")
    kfac.kfac_segments(c, choice, 6, order, offsets)
    assert int(offsets[6]) == 196 and order[196:].tolist() == [20, 21, 40, 41]
    rows, W, y = torch.randn(100, 8, device="cuda"), torch.randn(6, 4, 8, device="cuda"), torch.full((200, 4), 9.0, device="cuda")
    kfac.kfac_expert_forward(c, wl.fc_layer(1, 8, 4, 0), order, offsets, rows, W, y, fan=2)
    assert not y[20:22].any() and not y[40:42].any() and torch.isnan(gate[20]).all() and not gate[10].any()
    c.close()


def test_binding_refuses(ctx):
    r = kfac.router(8, 2)
    x, choice, gate = torch.zeros(4, 8, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    kfac.kfac_route(ctx, r, x, choice, gate)
    for bad in (dict(logits=x[:, :7]), dict(logits=x.half()), dict(logits=x.t().contiguous().t()), dict(choice=choice[:7]), dict(choice=choice.long()),
                dict(gate=gate.double()), dict(gate=gate[:3]), dict(bias=torch.zeros(7, device="cuda")), dict(logits=x.cpu()), dict(bias=torch.zeros(8))):
        with pytest.raises(ValueError):
            kfac.kfac_route(**{**dict(ctx=ctx, router=r, logits=x, choice=choice, gate=gate), **bad})
    with pytest.raises(kfac.KfacError):
        kfac.kfac_route(ctx, kfac.router(8, 9), x, torch.zeros(36, dtype=torch.int32, device="cuda"), torch.zeros(4, 9, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("E,groups,top,best", [(8, 1, 1, 1), (64, 8, 4, 2), (64, 8, 2, 1), (256, 8, 4, 2), (256, 1, 1, 1), (512, 8, 3, 2)])
def test_many_equal_ranks(ctx, E, groups, top, best, dtype):
    """Few different logits and biases: runs of equal ranks that reach over the last choice, with other ranks right behind them, and groups that are
    equal; every lane of the kernel may hold the largest one."""
    rng = np.random.default_rng(E + groups)
    n, fan = 600, min(7, top * E // groups)
    grid = rng.integers(0, 3, (n, E)) / 4.0
    grid[:100] = np.where(rng.random((100, E)) < 0.9, 0.5, 0.25)
    fine = grid + rng.integers(0, 2, (n, E)) * 2.0 ** -22           # (in fp32: neighbours that differ by a few of its steps)
    for logits in (grid, fine):
        for bias in (None, np.zeros(E), rng.integers(0, 2, E) * 0.25):
            for scores in (0, 1):
                _run(ctx, logits, bias, rng.standard_normal((n, fan)), dtype, 0, scores=scores, fan=fan, groups=groups, top_groups=top, group_best=best)


@pytest.mark.parametrize("scores", [0, 1])
def test_closed_by_the_lowest_value_of_the_type(ctx, scores):
    """Masks of -3.4e38 instead of -infinity: such experts are open, and come last."""
    rng = np.random.default_rng(12)
    for E in (16, 64, 256):
        logits = rng.standard_normal((80, E))
        logits[rng.random((80, E)) < 0.5] = -np.finfo(np.float32).max
        logits[0] = -np.finfo(np.float32).max
        logits[1, 3:] = -np.finfo(np.float32).max
        _run(ctx, logits, None, rng.standard_normal((80, 4)), F32, 0, scores=scores, fan=4, renormalise=scores == 0)
        _run(ctx, logits, 0.1 * rng.standard_normal(E), rng.standard_normal((80, 4)), F32, 0, scores=scores, fan=4, groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("scores", [0, 1])
@pytest.mark.parametrize("E", [16, 60, 256, 512])
@pytest.mark.parametrize("near", [2, 3, 5])
def test_near_ranks_around_the_last_choice(ctx, near, E, scores):
    """`near` experts whose ranks differ by less than fp32 resolves, by the rounding of a bias, with the last choice at every place among them: the
    first expert that is no choice takes the place of any choice that it beats in 64 bits; a closed one never does."""
    rng = np.random.default_rng(17 * near + E + scores)
    n = 90
    row = rng.standard_normal(E)
    top = rng.permutation(E)[:near + 3]                             # three clearly above, then the near ones
    row[top[:3]], row[top[3:]] = 3.0, 2.0 + 0.25 * rng.random(near)
    row = row.astype(np.float32).astype(np.float64)
    s = 1 / (1 + np.exp(-row)) if scores else np.exp(row - row.max()) / np.exp(row - row.max()).sum()
    bias = np.zeros(E)
    bias[top[:3]] = [2.0, 1.5, 1.0]
    bias[top[3:]] = 0.75 + s[top[3]] - s[top[3:]]                   # what fp32 keeps of it decides
    bias[[e for e in range(E) if e not in set(top)]] = -0.5
    logits = np.tile(row, (n, 1))
    logits[n // 3:, :] = np.where(np.isin(np.arange(E), top[:3]), logits[n // 3:, :], logits[n // 3:, :] + rng.integers(-2, 3, (n - n // 3, E)) * 2.0 ** -22)
    logits[-1, top[4:]] = -INF                                      # the neighbours of the last choice are closed
    for fan in range(3, min(E, near + 4)):
        for renormalise in (True, False):
            _run(ctx, logits, bias, rng.standard_normal((n, fan)), F32, 0, scores=scores, fan=fan, renormalise=renormalise)
