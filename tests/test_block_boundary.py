"""CPU-only: the entry points around the products of experts size their workspace and refuse bad arguments before touching the GPU."""
import ctypes

import pytest

from paper_2002_06015_amd import kfac, workloads as wl

INV, WS, OK = kfac.KFAC_ERR_INVALID, kfac.KFAC_ERR_WORKSPACE, kfac.KFAC_OK
P, Q, R, S, T, U, V, W = (ctypes.c_void_p(a << 36) for a in range(1, 9))     # made-up addresses, far apart, never dereferenced
at = ctypes.addressof
NAN, INF = float("nan"), float("inf")


def off(p, by):
    return ctypes.c_void_p(p.value + by)


@pytest.fixture()
def h():
    handle = ctypes.c_void_p()
    assert kfac.lib().kfac_create(at(handle), None, ctypes.c_void_p(0x100000), 256) == OK
    yield handle
    kfac.lib().kfac_destroy(handle)


def _call(fn, args, **change):
    values = dict(args)
    values.update(change)
    return getattr(kfac.lib(), fn)(*[v.value if isinstance(v, ctypes.c_void_p) else v for v in values.values()])


def _refuses(fn, ok, bad):
    for b in bad:
        assert _call(fn, ok, **b) == INV, b


def test_route_refuses(h):
    two = kfac.router(64, 2)
    ok = dict(ctx=h, router=at(two), n=8, type=0, logits=P, ld=64, bias=Q, choice=R, gate=S)
    routers = [kfac.router(0, 1), kfac.router(1025, 2), kfac.router(64, 0), kfac.router(64, 33), kfac.router(4, 5), kfac.router(64, 2, groups=0),
               kfac.router(64, 2, groups=6, top_groups=2), kfac.router(64, 2, groups=128), kfac.router(64, 2, groups=4, top_groups=5),
               kfac.router(64, 2, groups=4, top_groups=0), kfac.router(64, 9, groups=8, top_groups=1), kfac.router(64, 2, group_best=0),
               kfac.router(64, 2, group_best=3), kfac.router(64, 2, scores=2), kfac.router(64, 2, scores=-1), kfac.router(64, 2, renormalise=2),
               kfac.router(64, 2, scale=NAN), kfac.router(64, 2, scale=INF)]
    _refuses("kfac_route", ok, [dict(router=at(r)) for r in routers] + [
        dict(ctx=None), dict(router=None), dict(n=-1), dict(n=(1 << 29) + 1), dict(type=2), dict(logits=None), dict(ld=63), dict(ld=1 << 41),
        dict(choice=None), dict(gate=None), dict(logits=off(P, 2)), dict(type=1, logits=off(P, 1)), dict(bias=off(Q, 2)), dict(choice=off(R, 1)),
        dict(gate=off(S, 2)), dict(choice=P), dict(gate=P), dict(choice=Q), dict(gate=Q), dict(gate=R)])
    assert _call("kfac_route", ok, n=0, logits=None, choice=None, gate=None) == OK

    ok = dict(ctx=h, router=at(two), n=8, type=0, logits=P, ld=64, choice=R, dgate=S, dlogits=Q, ldd=64)
    _refuses("kfac_route_grad", ok, [dict(router=at(r)) for r in routers] + [
        dict(ctx=None), dict(router=None), dict(n=-1), dict(type=-1), dict(logits=None), dict(choice=None), dict(dgate=None), dict(dlogits=None), dict(ld=63),
        dict(ldd=63), dict(dlogits=off(Q, 2)), dict(dlogits=P), dict(dlogits=R), dict(dlogits=S), dict(choice=off(R, 2)), dict(dgate=off(S, 1))])
    assert _call("kfac_route_grad", ok, n=0, logits=None, choice=None, dgate=None, dlogits=None) == OK


def test_combine_refuses(h):
    ok = dict(ctx=h, n=8, fan=2, dim=16, type=0, y=P, ldy=16, gate=Q, out_type=1, residual=R, ldr=16, out=S, ldo=16)
    _refuses("kfac_combine", ok, [
        dict(ctx=None), dict(n=-2), dict(n=(1 << 30) + 2), dict(fan=0), dict(fan=3), dict(dim=0), dict(dim=(1 << 20) + 1), dict(type=2), dict(out_type=2),
        dict(y=None), dict(out=None), dict(ldy=15), dict(ldr=15), dict(ldo=15), dict(y=off(P, 2)), dict(out=off(S, 1)), dict(residual=off(R, 1)),
        dict(gate=off(Q, 2)), dict(out=P), dict(out=Q), dict(out=off(R, 32)), dict(out=R, ldo=17)])
    assert _call("kfac_combine", ok, n=0, y=None, gate=None, residual=None, out=None) == OK

    ok = dict(ctx=h, n=8, fan=2, dim=16, type=0, y=P, ldy=16, gate=Q, out_type=0, dout=R, ldd=16, dy=S, lddy=16, dgate=T)
    _refuses("kfac_combine_grad", ok, [
        dict(ctx=None), dict(n=-2), dict(fan=0), dict(fan=3), dict(dim=0), dict(type=2), dict(out_type=-1), dict(y=None), dict(dout=None),
        dict(dy=None, dgate=None), dict(ldy=15), dict(ldd=15), dict(lddy=15), dict(y=off(P, 2)), dict(dout=off(R, 2)), dict(dy=off(S, 2)),
        dict(gate=off(Q, 2)), dict(dgate=off(T, 2)), dict(dy=P), dict(dy=Q), dict(dy=R), dict(dy=T), dict(dgate=P), dict(dgate=Q), dict(dgate=R)])
    assert _call("kfac_combine_grad", ok, n=0, y=None, gate=None, dout=None) == OK


def test_keep_and_restore_refuse(h):
    ok = dict(ctx=h, rows=4, cols=40, type=0, x=P, ldx=40, q=Q, ldq=40, scales=R, lds=2)
    bad = [dict(ctx=None), dict(rows=-1), dict(rows=(1 << 40) + 1), dict(cols=-1), dict(cols=(1 << 30) + 1), dict(type=2), dict(x=None), dict(q=None), dict(scales=None),
           dict(ldx=39), dict(ldq=39), dict(lds=1), dict(x=off(P, 2))]
    _refuses("kfac_keep", ok, bad + [dict(q=P), dict(scales=P), dict(scales=Q)])
    assert _call("kfac_keep", ok, rows=0, x=None, q=None, scales=None) == OK and _call("kfac_keep", ok, cols=0, x=None, q=None, scales=None) == OK
    ok = dict(ctx=h, rows=4, cols=40, q=Q, ldq=40, scales=R, lds=2, type=0, x=P, ldx=40)
    _refuses("kfac_restore", ok, bad + [dict(x=Q), dict(x=R)])
    assert _call("kfac_restore", ok, rows=0, x=None, q=None, scales=None) == OK


def test_rms_norm_refuses(h):
    ok = dict(ctx=h, n=4, dim=40, type=1, x=P, ldx=40, stream=0, residual=Q, ldr=40, h=R, ldh=40, gamma=S, eps=1e-5, y=T, ldy=40, q=U, ldq=40, scales=V, lds=2)
    _refuses("kfac_rms_norm", ok, [
        dict(ctx=None), dict(n=-1), dict(n=(1 << 30) + 1), dict(dim=0), dict(dim=16385), dict(type=2), dict(stream=2), dict(x=None), dict(gamma=None),
        dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(residual=None), dict(h=None), dict(residual=None, h=None), dict(y=None, q=None, scales=None),
        dict(q=None), dict(scales=None), dict(ldx=39), dict(ldr=39), dict(ldh=39), dict(ldy=39), dict(ldq=39), dict(lds=1), dict(x=off(P, 1)),
        dict(residual=off(Q, 2)), dict(h=off(R, 2)), dict(gamma=off(S, 2)), dict(y=off(T, 1)), dict(h=P), dict(h=Q, ldh=41), dict(h=off(Q, 4)), dict(h=S),
        dict(h=T), dict(y=Q), dict(y=R), dict(y=S), dict(y=off(P, 2)), dict(y=P, ldy=41), dict(q=P), dict(q=Q), dict(q=R), dict(q=S), dict(q=T), dict(q=V),
        dict(scales=P), dict(scales=Q), dict(scales=R), dict(scales=S), dict(scales=T)])
    assert _call("kfac_rms_norm", ok, n=0, x=None, y=None) == OK

    assert kfac.kfac_rms_norm_workspace_bytes(-1, 8) == 0 and kfac.kfac_rms_norm_workspace_bytes(8, 0) == 0
    assert kfac.kfac_rms_norm_workspace_bytes(8, 16385) == 0 and kfac.kfac_rms_norm_workspace_bytes(0, 1) > 0
    ok = dict(ctx=h, n=4, dim=40, type=1, dy=P, lddy=40, stream=0, h=Q, ldh=40, gamma=R, eps=1e-5, dstream=S, ldr=40, dh=T, lddh=40, dgamma=U, decay=0.5, F=V)
    _refuses("kfac_rms_norm_grad", ok, [
        dict(ctx=None), dict(n=-1), dict(dim=0), dict(dim=16385), dict(type=2), dict(stream=-1), dict(dy=None), dict(h=None), dict(gamma=None),
        dict(eps=-1.0), dict(eps=NAN), dict(decay=1.0), dict(decay=-0.5), dict(decay=NAN), dict(dh=None, dgamma=None, F=None), dict(lddy=39), dict(ldh=39),
        dict(ldr=39), dict(lddh=39), dict(dy=off(P, 1)), dict(h=off(Q, 2)), dict(gamma=off(R, 2)), dict(dstream=off(S, 2)), dict(dh=off(T, 2)),
        dict(dgamma=off(U, 2)), dict(F=off(V, 2)), dict(dh=P), dict(dh=Q), dict(dh=R), dict(dh=off(S, 4)), dict(dh=S, lddh=41), dict(dgamma=P), dict(dgamma=Q),
        dict(dgamma=R), dict(dgamma=S), dict(dgamma=T), dict(dgamma=V), dict(F=P), dict(F=Q), dict(F=R), dict(F=S), dict(F=T)])
    assert _call("kfac_rms_norm_grad", ok) == WS                               # 256 bytes hold no sums of columns
    assert _call("kfac_rms_norm_grad", ok, n=0, dgamma=None, F=None) == OK


def test_workspaces_never_shrink():
    for f in (lambda n, d: kfac.kfac_rms_norm_workspace_bytes(n, d), lambda n, d: kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, d, 32), 4, n)):
        for d in (1, 31, 100, 2048, 2049, 4096, 4097, 8192, 8193, 16384):
            sizes = [f(n, d) for n in (0, 1, 2, 16, 17, 100, 2047, 2048, 2049, 10 ** 4, 10 ** 6)]
            assert sizes == sorted(sizes) and sizes[0] > 0
        for n in (1, 100, 2048, 5000, 10 ** 6):
            sizes = [f(n, d) for d in (1, 2, 31, 100, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16384)]
            assert sizes == sorted(sizes)
    sizes = [kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, 64, 32), 4, 960, fan) for fan in (6, 5, 4, 3, 2, 1)]
    assert sizes == sorted(sizes)


def test_kept_refuse(h):
    layer = kfac.kfac_layer(*wl.fc_layer(1, 64, 32))
    conv = kfac.kfac_layer(*wl.conv_layer(1, 64, 32, 3, 1, 1, 8))
    assert kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, 64, 32), 0, 8) == 0 and kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, 64, 32), 2, 8, 3) == 0
    assert kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, 64, 32), 2, -1) == 0 and kfac.kfac_kept_workspace_bytes(wl.fc_layer(1, 64, 32), 2, 8, 0) == 0
    o, f = ctypes.c_void_p(9 << 36), ctypes.c_void_p(10 << 36)
    shared = [dict(ctx=None), dict(L=None), dict(L=at(conv)), dict(experts=0), dict(n=-2), dict(type=2), dict(offsets=None), dict(offsets=off(f, 2)),
              dict(order=off(o, 2)), dict(fan=0), dict(fan=3), dict(q=None), dict(scales=None), dict(ldq=63), dict(lds=1)]
    ok = dict(ctx=h, L=at(layer), experts=4, n=8, fan=2, type=0, order=o, offsets=f, q=P, ldq=64, scales=Q, lds=2, dy=R, ldy=32, dW=S)
    _refuses("kfac_expert_grad_weight_kept", ok, shared + [dict(dy=None), dict(dW=None), dict(ldy=31), dict(dW=P), dict(dW=Q), dict(dW=R),
                                                           dict(dW=off(S, 2)), dict(dy=off(R, 2))])
    ok = dict(ctx=h, L=at(layer), experts=4, n=8, fan=2, type=0, order=o, offsets=f, q=P, ldq=64, scales=Q, lds=2, g=R, ldg=32, decay=0.5, A=S, G=T)
    _refuses("kfac_stats_expert_kept", ok, shared + [dict(g=None), dict(A=None, G=None), dict(ldg=31), dict(decay=1.0), dict(decay=NAN), dict(A=P), dict(A=Q),
                                                     dict(A=R), dict(A=T), dict(G=P), dict(G=Q), dict(G=R), dict(A=off(S, 2)), dict(G=off(T, 2))])
    assert _call("kfac_stats_expert_kept", ok, n=0) == OK
