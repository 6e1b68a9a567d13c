"""The join of the experts' results and its gradients on the GPU against their float64 definitions.

Tolerances: a sum of m fp32 terms is within (m + 4) 2^-24 of the sum of their magnitudes, an output in bf16 within 2^-8 of its value
besides, one in fp32 within 2^-24.  The sums of a gate's gradient are at most 8 ceil(dim / 512) terms in a thread, 6 steps in a wave, 3
over waves."""
import numpy as np
import pytest
import torch

from oracle import blocks as B
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


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


def _within(got, ref, mag, terms, dtype):
    assert (np.abs(_values(got) - ref) <= (terms + 4) * 2.0 ** -24 * mag + UNIT[dtype] * np.abs(ref) + 1e-40).all()


SHAPES = [  # tokens, fan, dim, pad
    (0, 2, 8, 0), (1, 1, 1, 0), (1, 2, 1024, 0), (4, 2, 1024, 0), (3, 3, 7, 0), (5, 1, 515, 3), (7, 5, 64, 1), (33, 8, 100, 8), (130, 4, 1001, 7), (64, 2, 2056, 0),
    (9, 32, 40, 0), (2, 2, 20001, 0), (4099, 2, 72, 0), (5000, 4, 600, 0), (4097, 1, 513, 1), (4100, 6, 1000, 0),
]


@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)], ids=["f32", "f32_bf16", "bf16_f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(str(v) for v in s) for s in SHAPES])
def test_combine(ctx, shape, types):
    tokens, fan, dim, pad = shape
    typ, out_type = types
    n = tokens * fan
    rng = np.random.default_rng(tokens + dim)
    y, _ = _rows(rng.standard_normal((n, dim)), typ, pad)
    r, _ = _rows(rng.standard_normal((tokens, dim)), out_type, pad)
    d, _ = _rows(rng.standard_normal((tokens, dim)), out_type, pad)
    gate = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda()
    g = gate.cpu().double().numpy()
    for weight, residual in ((gate, r), (None, None)):
        out, whole = _rows(np.zeros((tokens, dim)), out_type, pad, 5.0)
        kfac.kfac_combine(ctx, y, weight, out, residual=residual)
        torch.cuda.synchronize()
        ref, mag = B.combine(_values(y), None if weight is None else g, fan, None if residual is None else _values(r))
        _within(out, ref, mag, fan + 1, out_type)
        assert bool((whole[-1] == 5.0).all()) and bool((whole[:, dim:] == 5.0).all())
        dy, whole = _rows(np.zeros((n, dim)), typ, pad, 5.0)
        dgate = torch.full((n + 1,), 5.0, device="cuda")
        kfac.kfac_combine_grad(ctx, y, weight, d, dy, dgate[:n])
        torch.cuda.synchronize()
        refy, refg, magg = B.combine_grad(_values(y), None if weight is None else g, fan, _values(d))
        _within(dy, refy, np.abs(refy), 1, typ)
        _within(dgate[:n], refg, magg, 8 * ((dim + 511) // 512) + 10, F32)
        assert bool((whole[-1] == 5.0).all()) and bool((whole[:, dim:] == 5.0).all()) and float(dgate[n]) == 5.0
    if n:   # one of the two alone: the same bits, the other's tensors not touched
        alone, other = torch.empty_like(dgate[:n]), torch.empty_like(dy)
        kfac.kfac_combine_grad(ctx, y, None, d, None, alone)
        kfac.kfac_combine_grad(ctx, None, None, d, other, None)
        assert torch.equal(alone, dgate[:n]) and torch.equal(other, dy.contiguous())


def test_in_place_and_columns_of_one_tensor(ctx):
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    y, gate, wide = (torch.randn(*s, generator=g, device="cuda") for s in ((60, 40), (60,), (30, 100)))
    stream, out = wide[:, 3:43], torch.empty(30, 40, device="cuda")
    kfac.kfac_combine(ctx, y, gate, out, residual=stream)
    kfac.kfac_combine(ctx, y, gate, wide[:, 50:90], residual=stream)
    assert torch.equal(wide[:, 50:90], out)
    before = wide.clone()
    kfac.kfac_combine(ctx, y, gate, stream, residual=stream)
    assert torch.equal(stream, out) and torch.equal(wide[:, 43:], before[:, 43:]) and torch.equal(wide[:, :3], before[:, :3])


def test_sum_over_choices_is_the_gradient_of_the_rows(ctx):
    """kfac_expert_grad_input's dx, summed over a token's experts and added to the stream's gradient."""
    rng = np.random.default_rng(2)
    layer, E, tokens, fan = wl.fc_layer(1, 24, 40, 0), 5, 37, 2
    c = kfac.Context([layer], workspace_bytes=kfac.kfac_segments_workspace_bytes(74, E))
    choice = torch.from_numpy(rng.integers(0, E, tokens * fan).astype(np.int32)).cuda()
    order, offsets = torch.empty(74, dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    kfac.kfac_segments(c, choice, E, order, offsets)
    W, dy, ds = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((E, 40, 24), (74, 40), (tokens, 24)))
    dx, out = torch.empty(74, 24, device="cuda"), torch.empty(tokens, 24, device="cuda")
    kfac.kfac_expert_grad_input(c, layer, order, offsets, dy, W, dx)
    kfac.kfac_combine(c, dx, None, out, residual=ds)
    ref = ds.double() + torch.matmul(dy.double()[:, None, :], W.double()[choice.long()]).view(tokens, fan, 24).sum(1)
    mag = ds.double().abs() + torch.matmul(dy.double().abs()[:, None, :], W.double().abs()[choice.long()]).view(tokens, fan, 24).sum(1)
    assert bool(((out.double() - ref).abs() <= (40 + 12) * 2.0 ** -24 * mag).all())
    c.close()


def test_infinities_and_nan_stay_in_their_token(ctx):
    y, gate, out = torch.ones(6, 16, device="cuda"), torch.ones(6, device="cuda"), torch.empty(3, 16, device="cuda")
    y[2, 5], gate[4] = float("inf"), float("nan")
    kfac.kfac_combine(ctx, y, gate, out)
    assert torch.isinf(out[1, 5]) and torch.isnan(out[2]).all() and (out[0] == 2).all() and (out[1, :5] == 2).all()
    dy, dgate = torch.empty_like(y), torch.empty(6, device="cuda")
    kfac.kfac_combine_grad(ctx, y, gate, torch.ones(3, 16, device="cuda"), dy, dgate)
    assert torch.isinf(dgate[2]) and torch.isnan(dy[4]).all() and bool(torch.isfinite(dgate[[0, 1, 3, 4, 5]]).all()) and bool(torch.isfinite(dy[[0, 1, 2, 3, 5]]).all())


def test_binding_refuses(ctx):
    y, gate, out = torch.zeros(6, 16, device="cuda"), torch.zeros(6, device="cuda"), torch.zeros(3, 16, device="cuda")
    for bad in (dict(out=out[:, :15]), dict(out=torch.zeros(4, 16, device="cuda")), dict(gate=gate[:5]), dict(gate=gate.half()), dict(residual=out.bfloat16()),
                dict(y=y.half()), dict(out=out.cpu()), dict(residual=out[:2])):
        with pytest.raises(ValueError):
            kfac.kfac_combine(**{**dict(ctx=ctx, y=y, gate=gate, out=out), **bad})
    for bad in (dict(dy=None, dgate=None), dict(y=None), dict(dy=y.bfloat16()), dict(dgate=gate[:5])):
        with pytest.raises(ValueError):
            kfac.kfac_combine_grad(**{**dict(ctx=ctx, y=y, gate=gate, dout=out, dy=torch.zeros_like(y), dgate=gate.clone()), **bad})


def test_tokens_without_choices_are_refused(ctx):
    """Nothing would be written for them; no tokens at all are fine."""
    none, out = torch.empty(0, 8, device="cuda"), torch.full((5, 8), 3.0, device="cuda")
    with pytest.raises(ValueError):
        kfac.kfac_combine(ctx, none, None, out, residual=torch.zeros(5, 8, device="cuda"))
    with pytest.raises(ValueError):
        kfac.kfac_combine_grad(ctx, None, None, out, none, None)
    kfac.kfac_combine(ctx, none, None, none.clone())
    kfac.kfac_combine_grad(ctx, None, None, none, none.clone(), None)
    assert bool((out == 3.0).all())
