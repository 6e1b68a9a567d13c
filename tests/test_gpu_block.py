"""Norm, routing, experts, join and kept activations as one layer uses them: gradients against automatic differentiation in float64, the same
bits from a captured graph, contexts on several streams, offsets beyond 2^31."""
import numpy as np
import pytest
import torch

from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


class Block:
    """out = h + sum_j gate_j W_{e_j} y,  y = norm of h = x + residual, logits = y Wr."""

    def __init__(self, tokens, dim, E, fan, typ, stream, seed=0, kept=True):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.shape, self.kept = (tokens, dim, E, fan), kept
        self.layer, self.router, n = wl.fc_layer(1, dim, dim, 0), kfac.router(E, fan, scores=kfac.KFAC_ROUTE_SIGMOID, scale=1.5), tokens * fan
        self.x, self.residual, self.dout = rand(tokens, dim).to(typ), rand(tokens, dim).to(stream), rand(tokens, dim).to(stream)
        self.gamma, self.Wr, self.W = 1 + 0.2 * rand(dim), rand(dim, E) / dim ** 0.5, (rand(E, dim, dim) / dim ** 0.5).to(typ)
        self.bias = 0.05 * rand(E)
        new = lambda *s, dtype=F32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.h, self.y, self.logits = new(tokens, dim, dtype=stream), new(tokens, dim, dtype=typ), new(tokens, E)
        self.q, self.scales = new(tokens, dim, dtype=E4M3), new(tokens, (dim + 31) // 32, dtype=torch.uint8)
        self.choice, self.gate = new(n, dtype=torch.int32), new(tokens, fan)
        self.order, self.offsets = new(n, dtype=torch.int32), new(E + 1, dtype=torch.int32)
        self.results, self.out = new(n, dim, dtype=typ), new(tokens, dim, dtype=stream)
        self.dresults, self.dgate, self.dlogits, self.dchoice = new(n, dim, dtype=typ), new(tokens, fan), new(tokens, E), new(n, dim, dtype=typ)
        self.dW, self.dy, self.dh = new(E, dim, dim), new(tokens, dim, dtype=typ), new(tokens, dim, dtype=stream)
        self.dgamma, self.F, self.A, self.G = new(dim), torch.zeros(dim, device="cuda"), torch.zeros(E, dim, dim, device="cuda"), torch.zeros(E, dim, dim, device="cuda")
        self.dyr, self.dWr = new(tokens, dim), new(dim, E)
        self.need = max(kfac.kfac_segments_workspace_bytes(n, E), kfac.kfac_expert_workspace_bytes(self.layer, E, n),
                        kfac.kfac_kept_workspace_bytes(self.layer, E, n, fan), kfac.kfac_rms_norm_workspace_bytes(tokens, dim))
        self.ctx = kfac.Context([self.layer], workspace_bytes=self.need)

    def run(self, ctx=None):
        c, k, fan = ctx or self.ctx, kfac, self.shape[3]
        k.kfac_rms_norm(c, self.x, self.gamma, 1e-5, self.y, residual=self.residual, h=self.h, q=self.q, scales=self.scales)
        torch.mm(self.y.float(), self.Wr, out=self.logits)
        k.kfac_route(c, self.router, self.logits, self.choice, self.gate, bias=self.bias)
        k.kfac_segments(c, self.choice, self.shape[2], self.order, self.offsets)
        k.kfac_expert_forward(c, self.layer, self.order, self.offsets, self.y, self.W, self.results, fan=fan)
        k.kfac_combine(c, self.results, self.gate, self.out, residual=self.h)
        k.kfac_combine_grad(c, self.results, self.gate, self.dout, self.dresults, self.dgate)
        k.kfac_route_grad(c, self.router, self.logits, self.choice, self.dgate, self.dlogits)
        k.kfac_expert_grad_input(c, self.layer, self.order, self.offsets, self.dresults, self.W, self.dchoice)
        if self.kept:
            k.kfac_expert_grad_weight_kept(c, self.layer, self.order, self.offsets, self.q, self.scales, self.dresults, self.dW, fan=fan)
            k.kfac_stats_expert_kept(c, self.layer, self.order, self.offsets, self.q, self.scales, self.dresults, 0.9, self.A, self.G, fan=fan)
        else:
            k.kfac_expert_grad_weight(c, self.layer, self.order, self.offsets, self.y, self.dresults, self.dW, fan=fan)
        torch.mm(self.dlogits, self.Wr.t(), out=self.dyr)
        torch.mm(self.y.float().t(), self.dlogits, out=self.dWr)
        self.dyr_t = self.dyr.to(self.y.dtype)
        k.kfac_combine(c, self.dchoice, None, self.dy, residual=self.dyr_t)
        k.kfac_rms_norm_grad(c, self.dy, self.h, self.gamma, 1e-5, self.dh, dstream=self.dout, dgamma=self.dgamma, F=self.F, decay=0.9)

    def outputs(self):
        names = ["h", "y", "choice", "gate", "order", "offsets", "results", "out", "dresults", "dgate", "dlogits", "dchoice", "dW", "dy", "dh", "dgamma", "F", "A", "G",
                 "scales"]
        return {n: getattr(self, n).clone() for n in names} | {"q": self.q.view(torch.uint8).clone()}


def _gradients(b):
    """Automatic differentiation in float64 on the CPU, with the choices that were made."""
    tokens, dim, E, fan = b.shape
    f64 = lambda t: t.detach().double().cpu()  # noqa: E731
    x, gamma, W, Wr = (f64(t).requires_grad_() for t in (b.x, b.gamma, b.W, b.Wr))
    h = x + f64(b.residual)
    y = gamma * h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    logits = y @ Wr
    choice = b.choice.cpu().long().view(tokens, fan)
    s = torch.sigmoid(logits).gather(1, choice)
    gate = 1.5 * s / s.sum(1, keepdim=True)
    out = h + sum(gate[:, j:j + 1] * torch.stack([W[choice[t, j]] @ y[t] for t in range(tokens)]) for j in range(fan))
    (out * f64(b.dout)).sum().backward()
    return {"out": out.detach(), "dh": x.grad, "dgamma": gamma.grad, "dW": W.grad, "dWr": Wr.grad}


def test_gradients():
    """fp32: within 2e-5 of the largest element (sums of at most 300 terms through five operators, each with a relative error below 1e-6;
    the margin is for the cancellation in them); weights from inputs in 8 bits: every input within 2^-4, so a row of dW within
    2^-4 of the largest sum of magnitudes."""
    b = Block(150, 40, 5, 2, F32, F32, kept=False)
    b.run()
    want = _gradients(b)
    for name, ref in want.items():
        got = getattr(b, name).double().cpu()
        assert float((got - ref).abs().max()) <= 2e-5 * float(ref.abs().max()), name
    exact = b.dW.clone()
    b.kept = True
    b.run()
    e = b.choice.long().view(-1)
    mag = torch.stack([b.dresults.abs()[e == i].t() @ (b.y.abs() + 2.0 ** -6 * b.y.abs().amax()).repeat_interleave(2, 0)[e == i] for i in range(5)])
    assert bool(((b.dW - exact).abs() <= 2.0 ** -4 * mag + 1e-6).all()) and float((b.dW - exact).abs().max()) > 0


@pytest.mark.parametrize("typ,stream", [(F32, F32), (BF16, F32), (BF16, BF16)], ids=["f32", "bf16_f32", "bf16"])
def test_graph_gives_the_same_bits(typ, stream):
    b = Block(300, 72, 6, 2, typ, stream, seed=3)
    b.run()                                                                    # (libraries set up)
    b.F.zero_(), b.A.zero_(), b.G.zero_()
    b.run()
    eager = b.outputs()
    again = Block(300, 72, 6, 2, typ, stream, seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        c = kfac.Context([again.layer], workspace_bytes=again.need, stream=side)
        again.run(c)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            again.run(c)
    for replay in range(4):
        again.F.zero_(), again.A.zero_(), again.G.zero_()
        for name in ("choice", "gate", "out", "dh", "dW", "dlogits"):
            getattr(again, name).zero_()
        graph.replay()
        if replay % 2:
            torch.randn(1000, 1000, device="cuda").sum().item()              # the program's own work
        torch.cuda.synchronize()
        got = again.outputs()
        for name, v in eager.items():
            assert torch.equal(got[name], v), (replay, name)
    # other inputs of the same sizes
    other = Block(300, 72, 6, 2, typ, stream, seed=4)
    other.run()
    for name in ("x", "residual", "dout", "gamma", "Wr", "W", "bias"):
        getattr(again, name).copy_(getattr(other, name))
    again.F.zero_(), again.A.zero_(), again.G.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got, want = again.outputs(), other.outputs()
    assert all(torch.equal(got[name], want[name]) for name in want)


def test_two_contexts_on_two_streams():
    blocks = [Block(200, 64, 4, 2, BF16, F32, seed=i) for i in (5, 6)]
    for b in blocks:
        b.run()
        b.F.zero_(), b.A.zero_(), b.G.zero_()
        b.run()
    want = [b.outputs() for b in blocks]
    for b in blocks:
        b.F.zero_(), b.A.zero_(), b.G.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    contexts = []
    for b, s in zip(blocks, streams):
        with torch.cuda.stream(s):
            contexts.append(kfac.Context([b.layer], workspace_bytes=b.need, stream=s))
    torch.cuda.synchronize()
    for b, s, c in zip(blocks, streams, contexts):
        with torch.cuda.stream(s):
            b.run(c)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        got = b.outputs()
        assert all(torch.equal(got[name], w[name]) for name in w)


def test_offsets_beyond_31_bits():
    """Rows so far apart that their offsets, in elements and in bytes, pass 2^31."""
    far = (1 << 31) + 64
    room = torch.zeros(far + 64, dtype=torch.uint8, device="cuda")
    wide = lambda cols: torch.as_strided(room, (2, cols), (far, 1))  # noqa: E731
    ctx = kfac.Context([wl.fc_layer(1, 64, 32)], workspace_bytes=1 << 16)
    x = torch.randn(2, 48, device="cuda")
    q, s = torch.empty(2, 48, dtype=E4M3, device="cuda"), torch.empty(2, 2, dtype=torch.uint8, device="cuda")
    kfac.kfac_keep(ctx, x, q, s)
    kfac.kfac_keep(ctx, x, wide(48).view(E4M3), s)
    assert torch.equal(wide(48), q.view(torch.uint8))
    back, want = torch.empty(2, 48, device="cuda"), torch.empty(2, 48, device="cuda")
    kfac.kfac_restore(ctx, wide(48).view(E4M3), s, back)
    kfac.kfac_restore(ctx, q, s, want)
    assert torch.equal(back, want)
    del room
    half = torch.zeros(far + 64, dtype=BF16, device="cuda")
    a = torch.as_strided(half, (2, 48), (far, 1))
    a.copy_(x)
    b, gamma = x.bfloat16(), torch.randn(48, device="cuda")
    y, y2 = torch.empty(2, 48, dtype=BF16, device="cuda"), torch.empty(2, 48, dtype=BF16, device="cuda")
    kfac.kfac_rms_norm(ctx, a, gamma, 1e-5, y)
    kfac.kfac_rms_norm(ctx, b, gamma, 1e-5, y2)
    assert torch.equal(y, y2)
    dh, dh2 = torch.empty_like(y), torch.empty_like(y)
    dg, dg2 = torch.empty(48, device="cuda"), torch.empty(48, device="cuda")
    kfac.kfac_rms_norm_grad(ctx, y, a, gamma, 1e-5, dh, dstream=a, dgamma=dg)
    kfac.kfac_rms_norm_grad(ctx, y, b, gamma, 1e-5, dh2, dstream=b, dgamma=dg2)
    assert torch.equal(dh, dh2) and torch.equal(dg, dg2)
    out, out2, gate = torch.empty(1, 48, device="cuda"), torch.empty(1, 48, device="cuda"), torch.randn(2, device="cuda")
    kfac.kfac_combine(ctx, a, gate, out)
    kfac.kfac_combine(ctx, b, gate, out2)
    assert torch.equal(out, out2)
    d, d2 = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    kfac.kfac_combine_grad(ctx, a, gate, out, None, d)
    kfac.kfac_combine_grad(ctx, b, gate, out, None, d2)
    assert torch.equal(d, d2)
    r = kfac.router(48, 3)
    c, c2, g, g2 = (torch.empty(6, dtype=t, device="cuda") for t in (torch.int32, torch.int32, F32, F32))
    kfac.kfac_route(ctx, r, a, c, g.view(2, 3))
    kfac.kfac_route(ctx, r, b, c2, g2.view(2, 3))
    assert torch.equal(c, c2) and torch.equal(g, g2)
    dl = torch.empty(2, 48, dtype=BF16, device="cuda")
    kfac.kfac_route_grad(ctx, r, b, c, g.view(2, 3), dl)
    kfac.kfac_route_grad(ctx, r, b, c, g.view(2, 3), a)
    assert torch.equal(a, dl)
    ctx.close()


def test_other_device_is_refused():
    ctx = kfac.Context([wl.fc_layer(1, 8, 8)], workspace_bytes=256)
    with pytest.raises(ValueError):
        kfac.kfac_keep(ctx, torch.zeros(2, 8), torch.zeros(2, 8, dtype=torch.uint8).view(E4M3), torch.zeros(2, 1, dtype=torch.uint8))
    ctx.close()


def test_profile_names_the_launches():
    b = Block(64, 40, 4, 2, F32, F32)
    kfac.kfac_profile_enable(b.ctx, True)
    b.run()
    seen = [(e["kernel"], e["variant"]) for e in kfac.kfac_profile_read(b.ctx)]
    kfac.kfac_profile_enable(b.ctx, False)
    for want in (("norm", 0), ("route", 0), ("combine", 0), ("combine", 1), ("route", 1), ("expert", 2), ("expert", 3), ("norm", 1), ("norm", 2)):
        assert want in seen, want
    assert np.isfinite([b.dh.abs().max().item()]).all()


@pytest.mark.parametrize("typ", [F32, BF16], ids=["f32", "bf16"])
def test_padded_batch(typ):
    """Tokens whose logits are all -infinity, in the middle, as whole runs and at the end: their rows are the residual's alone, and the experts' gradients
    and factors are those of the batch without them (sums in fp32 of at most `rows` terms in two orders: rows 2^-23 of the sum of magnitudes)."""
    T, dim, E, fan = 190, 72, 5, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    pad = torch.zeros(T, dtype=torch.bool, device="cuda")
    pad[7], pad[50:90], pad[150:] = True, True, True
    h, logits, dout, W = rand(T, dim).to(typ), rand(T, E), rand(T, dim).to(typ), (rand(E, dim, dim) / 8).to(typ)
    logits[pad] = -float("inf")
    layer, router = wl.fc_layer(1, dim, dim, 0), kfac.router(E, fan)
    got = []
    for rows in (slice(None), ~pad):
        x, l, d = h[rows].contiguous(), logits[rows].contiguous(), dout[rows].contiguous()
        t = len(x)
        n = t * fan
        new = lambda *s, dtype=F32: torch.full(s, 7, dtype=dtype, device="cuda")  # noqa: E731
        need = max(kfac.kfac_segments_workspace_bytes(n, E), kfac.kfac_expert_workspace_bytes(layer, E, n), kfac.kfac_kept_workspace_bytes(layer, E, n, fan))
        c = kfac.Context([layer], workspace_bytes=need)
        q, s = torch.empty(t, dim, dtype=E4M3, device="cuda"), new(t, (dim + 31) // 32, dtype=torch.uint8)
        choice, gate, order, offsets = new(n, dtype=torch.int32), new(t, fan), new(n, dtype=torch.int32), new(E + 1, dtype=torch.int32)
        y, out, dy, dgate, dl, dx = new(n, dim, dtype=typ), new(t, dim, dtype=typ), new(n, dim, dtype=typ), new(t, fan), new(t, E), new(n, dim, dtype=typ)
        dW, A, G = new(E, dim, dim), new(E, dim, dim), new(E, dim, dim)
        kfac.kfac_keep(c, x, q, s)
        kfac.kfac_route(c, router, l, choice, gate)
        kfac.kfac_segments(c, choice, E, order, offsets)
        kfac.kfac_expert_forward(c, layer, order, offsets, x, W, y, fan=fan)
        kfac.kfac_combine(c, y, gate, out, residual=x)
        kfac.kfac_combine_grad(c, y, gate, d, dy, dgate)
        kfac.kfac_route_grad(c, router, l, choice, dgate, dl)
        kfac.kfac_expert_grad_input(c, layer, order, offsets, dy, W, dx)
        kfac.kfac_expert_grad_weight_kept(c, layer, order, offsets, q, s, dy, dW, fan=fan)
        kfac.kfac_stats_expert_kept(c, layer, order, offsets, q, s, dy, 0.0, A, G, fan=fan)
        values = new(t, dim)
        kfac.kfac_restore(c, q, s, values)
        torch.cuda.synchronize()
        got.append(dict(choice=choice.view(t, fan), gate=gate, out=out, dgate=dgate, dl=dl, dx=dx.view(t, fan, dim), y=y.view(t, fan, dim), dy=dy.view(t, fan, dim),
                        dW=dW, A=A, G=G, values=values, offsets=offsets))
        c.close()
    whole, real = got
    assert bool((whole["choice"][pad] == -1).all()) and torch.equal(whole["offsets"], real["offsets"])
    assert torch.equal(whole["out"][pad], h[pad])
    for name in ("gate", "y", "dy", "dgate", "dl", "dx"):
        assert bool((whole[name][pad] == 0).all()), name
    for name in ("choice", "gate", "dy"):
        assert torch.equal(whole[name][~pad], real[name]), name
    e = real["choice"].long()
    for i in range(E):
        at, j = (e == i).nonzero(as_tuple=True)
        v, d = real["values"][at].abs().double(), real["dy"][at, j].abs().double()
        for name, mag in (("dW", d.t() @ v), ("A", v.t() @ v / len(at)), ("G", d.t() @ d / len(at))):
            assert bool(((whole[name][i].double() - real[name][i].double()).abs() <= len(at) * 2.0 ** -23 * mag + 1e-30).all()), (name, i)
