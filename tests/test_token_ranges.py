"""CPU-only: what the token and expert entry points accept and refuse at the ends of their ranges."""
import ctypes

import pytest

from paper_2002_06015_amd import kfac, workloads as wl

INV, WS = kfac.KFAC_ERR_INVALID, kfac.KFAC_ERR_WORKSPACE
P, Q, R, S = ((a << 44) for a in (1, 2, 3, 4))     # made-up addresses, 16 TiB apart, never dereferenced


@pytest.fixture()
def h():
    handle = ctypes.c_void_p()
    assert kfac.lib().kfac_create(ctypes.addressof(handle), None, ctypes.c_void_p(0x100000), 256) == kfac.KFAC_OK
    yield handle.value
    kfac.lib().kfac_destroy(handle)


def test_distances_of_rows_that_no_tensor_has(h):
    """Rows times their distance beyond 2^40 elements are refused: products of the two that pass 64 bits among them."""
    far = (1 << 40) - 8
    embedding = lambda n, vocab, ldt, ldo: kfac.lib().kfac_embedding(h, n, P, 64, vocab, 16, 0, Q, ldt, 1.0, 0, R, ldo)  # noqa: E731
    assert embedding(8, 1 << 29, far, 16) == INV and embedding(1 << 29, 10, 16, far) == INV
    assert embedding(8, 1 << 24, 1 << 17, 16) == INV and embedding(8, 1 << 23, 1 << 40, 16) == INV and embedding(1 << 24, 10, 16, 1 << 17) == INV
    grad = lambda n, ld: kfac.lib().kfac_embedding_grad(h, n, P, 64, 10, 16, 0, Q, ld, 1.0, 0, R, 0.5, S)  # noqa: E731
    assert grad(1 << 29, far) == INV and grad(1 << 24, 1 << 17) == INV
    assert grad(1, far) == WS and grad(1 << 20, 1 << 20) == WS                  # no reason to refuse these: 256 bytes hold no lists


def test_columns_that_overlap_are_refused(h):
    """Views of one tensor whose columns meet, or whose rows lie differently far apart."""
    L = ctypes.addressof(kfac.kfac_layer(*wl.fc_layer(1, 16, 16)))
    dropout = lambda y, ldy=64, x=P, ldx=64: kfac.lib().kfac_dropout(h, 4, 16, 0, x, ldx, None, 0, 0.1, 1, 2, y, ldy)  # noqa: E731
    for at in (4, 60, 64 * 4 - 4, 64 * 4 + 4, 2 * 64 * 4 - 60):                 # bytes: rows are 256 bytes apart and 64 long
        assert dropout(P + at) == INV and dropout(P, x=P + at) == INV, at
    assert dropout(P + 64, ldy=65) == INV and dropout(P + 64, ldy=16) == INV
    forward = lambda y, x=P, W=Q: kfac.lib().kfac_expert_forward(h, L, 2, 8, 1, 0, None, S, x, 64, W, 64, y, 64)  # noqa: E731
    for at in (4, 60, 252, 260):
        assert forward(P + at) == INV and forward(Q + at) == INV and forward(P, x=P + at) == INV, at
    # a list of ids inside the rows of the output, and one that is longer than what lies between them
    lookup = lambda ids, n: kfac.lib().kfac_embedding(h, n, ids, 64, 10, 16, 0, Q, 16, 1.0, 0, R, 64)  # noqa: E731
    assert lookup(R + 32, 8) == INV and lookup(R + 64, 40) == INV


def test_workspace_of_experts_that_the_calls_refuse():
    """No size for what no call of the experts takes: layers that are not fully connected, more tiles than a launch has."""
    size = kfac.kfac_expert_workspace_bytes
    assert size(wl.fc_layer(1, 64, 32), 4, 100) > 0 and size(wl.fc_layer(1, 64, 32, 1), 1 << 16, 0) > 0
    assert size(wl.conv_layer(1, 64, 32, 3, 1, 1, 8), 4, 100) == 0 and size(wl.conv_layer(1, 64, 32, 1, 1, 0, 8), 4, 100) == 0
    assert size(wl.fc_layer(1, 64, 1 << 20), 1 << 16, 1 << 30) == 0
