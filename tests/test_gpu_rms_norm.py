"""The root-mean-square norm of a stream and its gradients on the GPU against their float64 definitions.

Tolerances: a row's sums are at most 32 terms in a thread, 6 steps in a wave, 16 over waves, so a mean is within 58 2^-24 of its terms'
magnitudes and 1 / sqrt(mean + eps) within 32 2^-24; with the products behind it 40 (y, u), 140 (gradients, of the magnitudes that are
added up).  Sums over n tokens: n + 140 at most.  An output in bf16 is within 2^-8 of its value besides, one in fp32 within 2^-24; 8 bits within
2^-4 of the value or 2^-10 of the scale."""
import numpy as np
import pytest
import torch

from oracle import blocks as B
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


def _ctx(n, dim):
    return kfac.Context([wl.fc_layer(2, 64, 32)], workspace_bytes=kfac.kfac_rms_norm_workspace_bytes(n, dim))


def _rows(a, dtype, pad=0, fill=float("nan")):
    t = torch.full((a.shape[0] + 1, a.shape[1] + pad), fill, dtype=dtype, device="cuda")
    t[:-1, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t[:-1, :a.shape[1]], t


def _bytes(n, dim, pad):
    q = torch.full((n + 1, dim + pad), 7, dtype=torch.uint8, device="cuda")
    s = torch.full((n + 1, (dim + 31) // 32 + pad), 9, dtype=torch.uint8, device="cuda")
    return q.view(torch.float8_e4m3fn)[:n, :dim], s[:n, :(dim + 31) // 32], q, s


def _values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _clean(whole, cols, mark=5.0):
    return bool((whole[-1] == mark).all()) and bool((whole[:, cols:] == mark).all())


SHAPES = [  # tokens, dim, pad
    (0, 8, 0), (1, 1, 0), (1, 31, 0), (2, 33, 0), (3, 7, 1), (4, 1024, 0), (5, 512, 0), (6, 513, 3), (17, 1025, 0), (33, 1001, 7), (3, 2048, 0), (9, 2049, 1), (130, 96, 8),
    (2, 4096, 0), (3, 4097, 3), (2, 8192, 0), (5, 8200, 0), (2, 16384, 0), (1, 16383, 0), (3000, 64, 0), (2500, 600, 0), (600, 5000, 0), (4200, 2056, 0),
]


@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)], ids=["f32", "f32_bf16", "bf16_f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(str(v) for v in s) for s in SHAPES])
def test_norm_and_gradients(shape, types):
    n, dim, pad = shape
    typ, stream = types
    rng = np.random.default_rng(n + dim)
    eps = 1e-5
    x, _ = _rows(rng.standard_normal((n, dim)), typ, pad)
    res, _ = _rows(10 * rng.standard_normal((n, dim)), stream, pad)
    gamma = torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda()
    gm = gamma.cpu().double().numpy()
    h, hw = _rows(np.zeros((n, dim)), stream, pad, 5.0)
    y, yw = _rows(np.zeros((n, dim)), typ, pad, 5.0)
    q, s, qw, sw = _bytes(n, dim, pad)
    ctx = _ctx(n, dim)
    kfac.kfac_rms_norm(ctx, x, gamma, eps, y, residual=res, h=h, q=q, scales=s)
    torch.cuda.synchronize()
    total = _values(x) + _values(res)
    hv = _values(h)
    assert (np.abs(hv - total) <= UNIT[stream] * np.abs(total) + U * (np.abs(_values(x)) + np.abs(_values(res)))).all()
    ref, _ = B.rms_norm(hv, gm, eps)
    assert (np.abs(_values(y) - ref) <= (40 * U + UNIT[typ]) * np.abs(ref)).all()
    assert _clean(hw, dim) and _clean(yw, dim)
    # eight bits: of y before its rounding
    scales = s.cpu().numpy()
    held = B.restore(q.view(torch.uint8).cpu().numpy(), scales)
    _, want = B.keep(ref)
    power = 2.0 ** (scales.astype(float) - 127)
    high = np.array([[np.abs(ref[i, 32 * b:32 * b + 32]).max() for b in range(scales.shape[1])] for i in range(n)]).reshape(scales.shape)
    near = np.abs(high / (448 * power) - 1) < 1e-5, np.abs(high / (224 * power) - 1) < 1e-5
    assert ((scales == want) | near[0] | near[1]).all()
    spread = np.repeat(power, 32, 1)[:, :dim]
    assert (np.abs(held - ref) <= (2.0 ** -4 + 41 * U) * np.abs(ref) + 2.0 ** -10 * spread).all()
    assert _clean(qw, dim, 7) and _clean(sw, (dim + 31) // 32, 9)
    # without 8 bits and without the type's output: the same bits
    alone, bytes_alone, scales_alone = torch.empty(n, dim, dtype=typ, device="cuda"), torch.empty(n, dim, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty_like(s)
    other = torch.empty(n, dim, dtype=stream, device="cuda")
    kfac.kfac_rms_norm(ctx, x, gamma, eps, alone, residual=res, h=other)
    kfac.kfac_rms_norm(ctx, x, gamma, eps, None, residual=res, h=other, q=bytes_alone, scales=scales_alone)
    assert torch.equal(alone, y.contiguous()) and torch.equal(other, h.contiguous())
    assert torch.equal(bytes_alone.view(torch.uint8), qw[:n, :dim].contiguous()) and torch.equal(scales_alone, s.contiguous())

    dy, _ = _rows(rng.standard_normal((n, dim)), typ, pad)
    ds, _ = _rows(rng.standard_normal((n, dim)), stream, pad)
    F0 = rng.random(dim).astype(np.float32)
    for dstream, decay in ((ds, 0.0), (None, 0.9)):
        dh, dw = _rows(np.zeros((n, dim)), stream, pad, 5.0)
        sums = torch.full((2 * dim + 2,), 5.0, device="cuda")
        F = torch.from_numpy(F0 if decay else F0 * np.float32("nan")).cuda()
        if n == 0:
            F = torch.from_numpy(F0).cuda()
        kfac.kfac_rms_norm_grad(ctx, dy, h, gamma, eps, dh, dstream=dstream, dgamma=sums[:dim], F=F, decay=decay)
        torch.cuda.synchronize()
        rd, md, rg, mg, rF = B.rms_norm_grad(_values(dy), hv, gm, eps, None if dstream is None else _values(dstream))
        assert (np.abs(_values(dh) - rd) <= 140 * U * md + UNIT[stream] * np.abs(rd) + 1e-40).all()
        assert (np.abs(_values(sums[:dim]) - rg) <= (n + 140) * U * mg).all()
        d = float(np.float32(decay))
        assert (np.abs(_values(F) - (d * F0 + (1 - d) * rF if n else F0)) <= (n + 180) * U * (d * F0 + rF)).all()
        assert _clean(dw, dim) and bool((sums[dim:] == 5.0).all())
        only = torch.empty(n, dim, dtype=stream, device="cuda")
        kfac.kfac_rms_norm_grad(ctx, dy, h, gamma, eps, only, dstream=dstream)          # no workspace, the same rows
        assert torch.equal(only, dh.contiguous())
        dg = torch.empty(dim, device="cuda")
        kfac.kfac_rms_norm_grad(ctx, dy, h, gamma, eps, None, dgamma=dg)
        assert torch.equal(dg, sums[:dim])
    ctx.close()


@pytest.mark.parametrize("typ", [F32, BF16], ids=["f32", "bf16"])
def test_without_a_residual_and_in_place(typ):
    rng = np.random.default_rng(1)
    ctx = _ctx(40, 300)
    x, _ = _rows(rng.standard_normal((40, 300)), typ, 4)
    gamma = torch.from_numpy(rng.standard_normal(300).astype(np.float32)).cuda()
    y = torch.empty(40, 300, dtype=typ, device="cuda")
    kfac.kfac_rms_norm(ctx, x, gamma, 1e-6, y)
    ref, _ = B.rms_norm(_values(x), gamma.cpu().double().numpy(), 1e-6)
    assert (np.abs(_values(y) - ref) <= (40 * U + UNIT[typ]) * np.abs(ref)).all()
    # the sum takes the residual's place, or x's; y takes x's
    res, _ = _rows(rng.standard_normal((40, 300)), typ, 4)
    h, want = torch.empty_like(y), torch.empty_like(y)
    kfac.kfac_rms_norm(ctx, x, gamma, 1e-6, want, residual=res, h=h)
    for which in range(3):
        a, b, o = x.clone(), res.clone(), torch.empty_like(y)
        kfac.kfac_rms_norm(ctx, a, gamma, 1e-6, a if which == 2 else o, residual=b, h=(b, a, b)[which])
        assert torch.equal((b, a, b)[which], h) and torch.equal(a if which == 2 else o, want)
    a = x.clone()
    kfac.kfac_rms_norm(ctx, a, gamma, 1e-6, a)
    assert torch.equal(a, y)
    dh = torch.empty_like(y)
    kfac.kfac_rms_norm_grad(ctx, y, h, gamma, 1e-6, dh, dstream=res)
    a, b = res.clone(), y.clone()
    kfac.kfac_rms_norm_grad(ctx, y, h, gamma, 1e-6, a, dstream=a)
    kfac.kfac_rms_norm_grad(ctx, b, h, gamma, 1e-6, b, dstream=res)
    assert torch.equal(a, dh) and torch.equal(b, dh)
    ctx.close()


def test_rows_of_zeros_and_values_that_are_not_finite():
    ctx = _ctx(6, 64)
    x = torch.ones(6, 64, device="cuda")
    x[0], x[1, 5], x[2, 40], x[3] = 0.0, float("nan"), float("inf"), 1e-30
    gamma, y = torch.ones(64, device="cuda"), torch.empty(6, 64, device="cuda")
    q, s = torch.empty(6, 64, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, 2, dtype=torch.uint8, device="cuda")
    kfac.kfac_rms_norm(ctx, x, gamma, 1e-5, y, q=q, scales=s)
    assert not y[0].any() and torch.isnan(y[1]).all() and bool((y[4:] == y[4, 0]).all())
    assert torch.isnan(y[2, 40]) and not y[2, :40].any()                   # the mean is infinite: the others are divided by it
    assert s[0].tolist() == [10, 10] and not q[0].float().any() and torch.isnan(q[1].float()).all() and torch.isnan(q[2, 40].float())
    kfac.kfac_rms_norm(ctx, x, gamma, 0.0, y)
    assert torch.isnan(y[0]).all()
    dh, dg = torch.empty(6, 64, device="cuda"), torch.empty(64, device="cuda")
    kfac.kfac_rms_norm_grad(ctx, torch.ones(6, 64, device="cuda"), x, gamma, 1e-5, dh, dgamma=dg)
    assert torch.isnan(dh[1]).all() and bool(torch.isfinite(dh[[0, 3, 4, 5]]).all()) and torch.isnan(dg[5])
    ctx.close()


def test_gradient_by_differences():
    """Central differences of a loss in float64 over the norm's output: steps of 2^-6 in h, |third derivative| below 40 / r^2."""
    rng = np.random.default_rng(3)
    ctx = _ctx(4, 48)
    h, gamma, dy = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((4, 48), (48,), (4, 48)))
    dh = torch.empty_like(h)
    kfac.kfac_rms_norm_grad(ctx, dy, h, gamma, 1e-3, dh)
    step, y = 2.0 ** -6, torch.empty_like(h)

    def loss(x):
        kfac.kfac_rms_norm(ctx, x, gamma, 1e-3, y)
        return (y.double() * dy.double()).sum(1)
    for c in range(0, 48, 5):
        e = torch.zeros_like(h)
        e[:, c] = step
        slope = (loss(h + e) - loss(h - e)) / (2 * step)
        # rounding of y: 48 terms of magnitude 10 at most, 2^-19 relative; curvature: step^2 / 6 of a third derivative of a few units
        assert float((slope - dh[:, c].double()).abs().max()) < 48 * 10 * 2.0 ** -19 / step + 10 * step ** 2
    ctx.close()


def test_refuses(gpu):
    ctx = kfac.Context([wl.fc_layer(2, 64, 32)], workspace_bytes=256)
    x, gamma, y = torch.zeros(4, 600, device="cuda"), torch.ones(600, device="cuda"), torch.zeros(4, 600, device="cuda")
    for bad in (dict(residual=x), dict(h=y), dict(q=torch.empty(4, 600, dtype=torch.float8_e4m3fn, device="cuda")), dict(gamma=gamma[:599]), dict(y=y.bfloat16()),
                dict(x=x.half()), dict(gamma=gamma.cpu()), dict(residual=x.clone(), h=y.bfloat16()), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            kfac.kfac_rms_norm(**{**dict(ctx=ctx, x=x, gamma=gamma, eps=1e-5, y=y), **bad})
    with pytest.raises(kfac.KfacError) as e:
        kfac.kfac_rms_norm_grad(ctx, x, y, gamma, 1e-5, None, dgamma=torch.empty(600, device="cuda"))
    assert e.value.status == kfac.KFAC_ERR_WORKSPACE
    ctx.close()
