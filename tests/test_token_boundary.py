"""CPU-only: the token and expert entry points size their workspace and refuse bad arguments before touching the GPU."""
import ctypes

import pytest

from paper_2002_06015_amd import kfac, workloads as wl

INV, WS = kfac.KFAC_ERR_INVALID, kfac.KFAC_ERR_WORKSPACE
P, Q, R, S = (ctypes.c_void_p(a << 32) for a in (1, 2, 3, 4))     # made-up addresses, far apart, never dereferenced


@pytest.fixture()
def h():
    handle = ctypes.c_void_p()
    assert kfac.lib().kfac_create(ctypes.addressof(handle), None, ctypes.c_void_p(0x100000), 256) == kfac.KFAC_OK
    yield handle
    kfac.lib().kfac_destroy(handle)


def _call(fn, args, **change):
    """The entry point with named arguments replaced."""
    values = dict(args)
    values.update(change)
    return getattr(kfac.lib(), fn)(*[v.value if isinstance(v, ctypes.c_void_p) else v for v in values.values()])


def test_workspace_sizes():
    assert kfac.kfac_segments_workspace_bytes(-1, 4) == 0 and kfac.kfac_segments_workspace_bytes(4, 0) == 0
    assert kfac.kfac_segments_workspace_bytes((1 << 30) + 1, 4) == 0 and kfac.kfac_segments_workspace_bytes(4, 1 << 30) == 0
    assert 0 < kfac.kfac_segments_workspace_bytes(0, 1) < kfac.kfac_segments_workspace_bytes(100000, 32000)
    assert kfac.kfac_embedding_workspace_bytes(8, 100, 0) == 0 and kfac.kfac_embedding_workspace_bytes(8, 0, 8) == 0
    assert kfac.kfac_embedding_workspace_bytes(8192, 32000, 64) < kfac.kfac_embedding_workspace_bytes(8192, 32000, 1024)
    layer = wl.fc_layer(1, 64, 32)
    assert kfac.kfac_expert_workspace_bytes(layer, 8, 100) > 0
    assert kfac.kfac_expert_workspace_bytes(layer, 0, 100) == 0 and kfac.kfac_expert_workspace_bytes(layer, 8, -1) == 0


def test_segments_refuses(h):
    ok = dict(ctx=h, n=8, ids=P, bits=32, num=4, order=Q, offsets=R)
    for bad in (dict(ctx=None), dict(n=-1), dict(n=(1 << 30) + 1), dict(num=0), dict(bits=16), dict(ids=None), dict(order=None), dict(offsets=None),
                dict(ids=ctypes.c_void_p((1 << 32) + 2)), dict(bits=64, ids=ctypes.c_void_p((1 << 32) + 4)), dict(order=P), dict(offsets=Q), dict(offsets=P)):
        assert _call("kfac_segments", ok, **bad) == INV, bad
    assert _call("kfac_segments", ok, n=100000) == WS


def test_embedding_refuses(h):
    ok = dict(ctx=h, n=8, ids=P, bits=64, vocab=10, dim=16, table_type=0, table=Q, ld_table=16, scale=1.0, out_type=1, out=R, ld_out=16)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(ctx=None), dict(n=-1), dict(bits=8), dict(vocab=0), dict(dim=0), dict(table_type=2), dict(out_type=-1), dict(ids=None), dict(table=None),
                dict(out=None), dict(ld_table=15), dict(ld_out=15), dict(scale=nan), dict(scale=inf), dict(out=Q), dict(out=P),
                dict(table=ctypes.c_void_p((2 << 32) + 2)), dict(out=ctypes.c_void_p((3 << 32) + 1))):
        assert _call("kfac_embedding", ok, **bad) == INV, bad
    assert _call("kfac_embedding", ok, n=0, ids=None, table=None, out=None) == kfac.KFAC_OK     # nothing to do

    ok = dict(ctx=h, n=8, ids=P, bits=64, vocab=10, dim=16, type=0, grad=Q, ld=16, scale=1.0, acc=0, dW=R, decay=0.5, A=S)
    for bad in (dict(ctx=None), dict(n=-1), dict(bits=8), dict(vocab=0), dict(dim=0), dict(type=2), dict(ids=None), dict(grad=None), dict(dW=None), dict(ld=15),
                dict(scale=nan), dict(decay=1.0), dict(decay=-0.1), dict(decay=nan), dict(dW=Q), dict(A=R), dict(A=Q), dict(A=P), dict(dW=P),
                dict(dW=ctypes.c_void_p((3 << 32) + 2)), dict(A=ctypes.c_void_p((4 << 32) + 2))):
        assert _call("kfac_embedding_grad", ok, **bad) == INV, bad
    assert _call("kfac_embedding_grad", ok) == WS                                               # 256 bytes hold no lists


def test_dropout_refuses(h):
    ok = dict(ctx=h, rows=4, cols=16, type=0, x=P, ldx=16, residual=Q, ldr=16, p=0.1, seed=1, offset=2, y=R, ldy=16)
    nan = float("nan")
    for bad in (dict(ctx=None), dict(rows=-1), dict(cols=-1), dict(rows=1 << 41), dict(type=3), dict(x=None), dict(y=None), dict(ldx=15), dict(ldr=15), dict(ldy=15),
                dict(p=-0.1), dict(p=1.1), dict(p=nan), dict(x=ctypes.c_void_p((1 << 32) + 2)), dict(y=ctypes.c_void_p((1 << 32) + 64)),
                dict(y=ctypes.c_void_p((2 << 32) + 64)), dict(y=P, ldy=17), dict(rows=1 << 30, cols=1 << 30, ldx=1 << 30, ldy=1 << 30, ldr=1 << 30)):
        assert _call("kfac_dropout", ok, **bad) == INV, bad
    assert _call("kfac_dropout", ok, rows=0, x=None, y=None) == kfac.KFAC_OK
    assert _call("kfac_dropout", ok, cols=0, x=None, y=None) == kfac.KFAC_OK


def test_experts_refuse(h):
    layer = kfac.kfac_layer(*wl.fc_layer(1, 64, 32))
    conv = kfac.kfac_layer(*wl.conv_layer(1, 64, 32, 3, 1, 1, 8))
    broken = kfac.kfac_layer(1, 0, 32, 1, 1, 0, 1, 1, 0)
    at = ctypes.addressof
    shared = (dict(ctx=None), dict(L=None), dict(L=at(conv)), dict(L=at(broken)), dict(experts=0), dict(experts=(1 << 16) + 1), dict(n=-2), dict(n=(1 << 30) + 2),
              dict(type=2), dict(offsets=None), dict(offsets=ctypes.c_void_p(0x502)), dict(order=ctypes.c_void_p(0x502)))
    o, f = ctypes.c_void_p(5 << 32), ctypes.c_void_p(6 << 32)

    ok = dict(ctx=h, L=at(layer), experts=4, n=8, fan=2, type=0, order=o, offsets=f, x=P, ldx=64, W=Q, ldw=65, y=R, ldy=32)
    for bad in shared + (dict(fan=0), dict(fan=3), dict(x=None), dict(W=None), dict(y=None), dict(ldx=63), dict(ldw=64), dict(ldy=31), dict(y=P), dict(y=Q),
                         dict(x=ctypes.c_void_p((1 << 32) + 2)), dict(n=1 << 30, fan=1, experts=1 << 16, L=at(kfac.kfac_layer(*wl.fc_layer(1, 64, 1 << 20))))):
        assert _call("kfac_expert_forward", ok, **bad) == INV, bad
    assert _call("kfac_expert_forward", ok, n=0, x=None, W=None, y=None) == kfac.KFAC_OK

    ok = dict(ctx=h, L=at(layer), experts=4, n=8, type=0, order=o, offsets=f, dy=P, ldy=32, W=Q, ldw=65, dx=R, ldx=64)
    for bad in shared + (dict(dy=None), dict(W=None), dict(dx=None), dict(ldx=63), dict(ldw=64), dict(ldy=31), dict(dx=P), dict(dx=Q)):
        assert _call("kfac_expert_grad_input", ok, **bad) == INV, bad
    assert _call("kfac_expert_grad_input", ok, n=0, dy=None, W=None, dx=None) == kfac.KFAC_OK

    ok = dict(ctx=h, L=at(layer), experts=4, n=8, fan=2, type=0, order=o, offsets=f, x=P, ldx=64, dy=Q, ldy=32, dW=R)
    for bad in shared + (dict(fan=0), dict(fan=3), dict(x=None), dict(dy=None), dict(dW=None), dict(ldx=63), dict(ldy=31), dict(dW=P), dict(dW=Q),
                         dict(dW=ctypes.c_void_p((3 << 32) + 2))):
        assert _call("kfac_expert_grad_weight", ok, **bad) == INV, bad

    ok = dict(ctx=h, L=at(layer), experts=4, n=8, fan=2, type=0, order=o, offsets=f, x=P, ldx=64, g=Q, ldg=32, decay=0.5, A=R, G=S)
    for bad in shared + (dict(fan=0), dict(fan=3), dict(x=None), dict(g=None), dict(A=None, G=None), dict(ldx=63), dict(ldg=31), dict(decay=1.0),
                         dict(decay=-1.0), dict(decay=float("nan")), dict(A=P), dict(G=Q), dict(A=S), dict(A=ctypes.c_void_p((3 << 32) + 2))):
        assert _call("kfac_stats_expert", ok, **bad) == INV, bad
    assert _call("kfac_stats_expert", ok, n=0) == kfac.KFAC_OK
