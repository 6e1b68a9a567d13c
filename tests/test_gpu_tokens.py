"""Segments, embedding and dropout on the GPU against their float64 definitions.

Tolerances: a sum of m fp32 terms is within (m + 4) 2^-24 of the sum of their magnitudes; an output in bf16 is within 2^-8 of its
value besides (round to nearest, 8 significant bits), one in fp32 within 2^-24; whole numbers and copies are exact."""
import numpy as np
import pytest
import torch

from oracle import tokens as T
from paper_2002_06015_amd import kfac, workloads as wl

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
LAYER = [wl.fc_layer(2, 64, 32)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    kfac.lib()


def _ctx(need=256):
    return kfac.Context(LAYER, workspace_bytes=max(256, need))


def _rows(a, dtype, pad=0, fill=float("nan")):
    """A device tensor with the values of `a`, rows `pad` elements further apart than they are long, `fill` between them."""
    t = torch.full((a.shape[0], a.shape[1] + pad), fill, dtype=dtype, device="cuda")
    t[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t[:, :a.shape[1]], t


def _values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------------------------------------------ segments
@pytest.mark.parametrize("bits", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,num", [(0, 1), (0, 600), (1, 1), (1, 40000), (63, 5), (64, 32), (65, 511), (1000, 512), (1025, 513), (8191, 70000),
                                   (8192, 16), (8193, 16), (20000, 511), (30000, 512), (50001, 70000), (300001, 3)])
def test_segments(n, num, bits):
    rng = np.random.default_rng(n + num)
    ids = rng.integers(-2, num + 2, n) if n % 2 else rng.integers(0, num, n)
    if n > 100:
        ids[10:60] = num // 2                                       # a run of equal ids
    order = torch.full((n + 3,), -7, dtype=torch.int32, device="cuda")
    offsets = torch.full((num + 4,), -7, dtype=torch.int32, device="cuda")
    ctx = _ctx(kfac.kfac_segments_workspace_bytes(n, num))
    kfac.kfac_segments(ctx, torch.from_numpy(ids).to(bits).cuda(), num, order[:n], offsets[:num + 1])
    torch.cuda.synchronize()
    ref_order, ref_offsets = T.segments(ids, num)
    assert np.array_equal(order.cpu().numpy(), np.concatenate([ref_order, [-7] * 3]))
    assert np.array_equal(offsets.cpu().numpy(), np.concatenate([ref_offsets, [-7] * 3]))
    ctx.close()


@pytest.mark.parametrize("n", [5000, 30000])
@pytest.mark.parametrize("ids", ["same", "none", "huge"])
def test_segments_of_one_id_and_of_none(n, ids):
    v = {"same": np.full(n, 4), "none": np.full(n, -1), "huge": np.full(n, 2 ** 40)}[ids].astype(np.int64)
    order, offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(8, dtype=torch.int32, device="cuda")
    ctx = _ctx(kfac.kfac_segments_workspace_bytes(n, 7))
    kfac.kfac_segments(ctx, torch.from_numpy(v).cuda(), 7, order, offsets)
    ref_order, ref_offsets = T.segments(v, 7)
    assert np.array_equal(order.cpu().numpy(), ref_order) and np.array_equal(offsets.cpu().numpy(), ref_offsets)
    ctx.close()


# ------------------------------------------------------------------------------------------------ embedding
@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,vocab,dim,pad", [(0, 3, 8, 0), (1, 1, 1, 0), (3, 7, 5, 0), (5, 9, 8, 3), (64, 100, 64, 0), (33, 50, 515, 1), (1000, 300, 1024, 8)])
def test_lookup(table, out, n, vocab, dim, pad):
    rng = np.random.default_rng(n + dim)
    ids = rng.integers(-1, vocab + 1, n)
    t, _ = _rows(rng.standard_normal((vocab, dim)), table, pad)
    o, whole = _rows(np.zeros((n, dim)), out, pad, 5.0)
    bits = torch.int32 if n % 2 else torch.int64
    ctx = _ctx()
    kfac.kfac_embedding(ctx, torch.from_numpy(ids).to(bits).cuda(), t, 1.7, o)
    ref = T.embedding(ids, _values(t), np.float64(np.float32(1.7)))
    assert np.all(np.abs(_values(o) - ref) <= (2.0 ** -24 + UNIT[out]) * np.abs(ref))
    assert bool((whole[:, dim:] == 5.0).all())
    ctx.close()


def test_lookup_beyond_32_bit_offsets():
    """Rows of a table of more than 2^32 elements."""
    vocab, dim = 70000, 65536
    table = torch.zeros(vocab, dim, dtype=BF16, device="cuda")
    table[vocab - 1] = torch.arange(dim, device="cuda").remainder(251).to(BF16)
    ids = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
    out = torch.full((3, dim), 7.0, dtype=BF16, device="cuda")
    ctx = _ctx()
    kfac.kfac_embedding(ctx, ids, table, 2.0, out)
    assert torch.equal(out[0].float(), 2 * torch.arange(dim, device="cuda").remainder(251).float()) and torch.equal(out[0], out[2])
    assert not bool(out[1].any())
    ctx.close()


def _zipf(rng, n, vocab):
    p = 1.0 / np.arange(1, vocab + 1)
    return rng.choice(rng.permutation(vocab), n, p=p / p.sum())


GRADS = [(0, 4, 8, "zipf"), (1, 1, 1, "zipf"), (7, 3, 5, "zipf"), (8, 20, 64, "zipf"), (9, 20, 515, "zipf"), (64, 1, 256, "same"), (1000, 2000, 100, "zipf"),
         (1000, 50, 1030, "none"), (8200, 70000, 32, "zipf"), (20000, 300, 64, "same"), (40000, 5000, 72, "zipf"), (40000, 11, 260, "runs")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim,kind", GRADS)
def test_embedding_grad(dtype, n, vocab, dim, kind):
    rng = np.random.default_rng(n + vocab + dim)
    ids = {"zipf": lambda: _zipf(rng, n, vocab), "same": lambda: np.full(n, vocab - 1), "none": lambda: np.full(n, vocab),
           "runs": lambda: np.sort(rng.integers(0, vocab, n))}[kind]().astype(np.int64)
    if n > 20 and kind == "zipf":
        ids[rng.integers(0, n, n // 10)] = -1
    pad, accumulate, decay = (3, True, 0.95) if n % 2 == 0 else (0, False, 0.0)
    g, _ = _rows(rng.standard_normal((n, dim)), dtype, pad)
    start, a0 = rng.standard_normal((vocab, dim)).astype(np.float32), rng.random(vocab).astype(np.float32)
    if not accumulate:
        start[:], a0[:] = np.nan, np.nan                          # never read
    buf = torch.full((vocab + 1, dim), 9.0, device="cuda")        # a row behind the end
    dW = buf[:vocab]
    dW.copy_(torch.from_numpy(start))
    A = torch.from_numpy(a0).cuda()
    d_ids = torch.from_numpy(ids).cuda()
    ctx = _ctx(kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
    kfac.kfac_embedding_grad(ctx, d_ids, g, 0.7, dW, accumulate, A, decay)
    ref, counts, mag = T.embedding_grad(ids, _values(g), np.float64(np.float32(0.7)), vocab)
    if accumulate:
        ref, mag = ref + start, mag + np.abs(start)
    err = np.abs(_values(dW) - ref)
    assert np.all(err <= (counts[:, None] + 4) * 2.0 ** -24 * mag)
    assert bool((buf[vocab] == 9.0).all())
    if n > 0:
        refA = np.float64(np.float32(decay)) * (a0 if decay else 0.0) + (1 - np.float64(np.float32(decay))) * counts / n
        assert np.allclose(_values(A), refA, rtol=8 * 2.0 ** -24, atol=0)
    else:
        assert np.array_equal(A.cpu().numpy(), a0, equal_nan=True)
    # the same bits again, and without the frequencies
    again = torch.from_numpy(start).cuda()
    kfac.kfac_embedding_grad(ctx, d_ids, g, 0.7, again, accumulate)
    assert torch.equal(again.view(torch.int32), dW.view(torch.int32))
    ctx.close()


def test_embedding_grad_by_differences():
    """The loss sum(out * R) is linear in the table: a difference quotient of the lookup is the gradient."""
    rng = np.random.default_rng(3)
    n, vocab, dim = 300, 40, 24
    ids = torch.from_numpy(_zipf(rng, n, vocab)).cuda()
    table, R = torch.from_numpy(rng.standard_normal((vocab, dim))).float().cuda(), torch.from_numpy(rng.standard_normal((n, dim))).float().cuda()
    out, dW = torch.empty(n, dim, device="cuda"), torch.empty(vocab, dim, device="cuda")
    ctx = _ctx(kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
    kfac.kfac_embedding_grad(ctx, ids, R, 3.0, dW)

    def loss(t):
        kfac.kfac_embedding(ctx, ids, t, 3.0, out)
        return float((out.double() * R.double()).sum())

    # h = 1: the rounding of n values of about 3 in fp32, each to 2^-24 of it, over 2 h
    for v in range(0, vocab, 7):
        for c in (0, 11, 23):
            step = torch.zeros_like(table)
            step[v, c] = 1.0
            want = (loss(table + step) - loss(table - step)) / 2
            assert abs(want - float(dW[v, c])) <= 2.0 ** -24 * n * 3 * 8
    ctx.close()


# ------------------------------------------------------------------------------------------------ dropout
def _dropped(rows, cols, dtype, p, pad=(0, 0, 0), residual=True, seed=(1 << 40) + 5, offset=3, poison=False):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, _ = _rows(rng.standard_normal((rows, cols)), dtype, pad[0])
    r, _ = _rows(rng.standard_normal((rows, cols)), dtype, pad[1]) if residual else (None, None)
    y, whole = _rows(np.zeros((rows, cols)), dtype, pad[2], 5.0)
    keep = T.dropout_keep(0, rows * cols, p, seed, offset).reshape(rows, cols)
    if poison:                                    # infinities and NaN where they are dropped
        x[torch.from_numpy(~keep).cuda()] = float("nan")
        x[0, 0] = float("inf") if not keep[0, 0] else x[0, 0]
    ctx = _ctx()
    kfac.kfac_dropout(ctx, x, p, seed, offset, y, residual=r)
    torch.cuda.synchronize()
    clean = np.where(keep, _values(x), 0.0)
    t = round(p * 65536)
    v = clean * (65536.0 / (65536.0 - t)) if t < 65536 else 0.0 * clean
    ref = v + (_values(r) if residual else 0.0)
    mag = np.abs(v) + (np.abs(_values(r)) if residual else 0.0)
    assert np.all(np.abs(_values(y) - ref) <= 4 * 2.0 ** -24 * mag + UNIT[dtype] * np.abs(ref))
    assert bool((whole[:, cols:] == 5.0).all())
    if not residual:
        assert np.array_equal(_values(y) != 0, keep & (_values(x) != 0))
    ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (3, 5), (4, 8), (9, 17), (5, 1001), (64, 24)])
@pytest.mark.parametrize("pad", [(0, 0, 0), (3, 1, 0), (8, 16, 8), (0, 0, 1)])
def test_dropout(dtype, rows, cols, pad):
    for p in (0.1, 0.5):
        _dropped(rows, cols, dtype, p, pad, residual=rows % 2 == 1)
    _dropped(rows, cols, dtype, 0.25, pad, residual=rows % 2 == 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_corners(dtype):
    for p in (0.0, 1e-7, 1.0, 0.99999):
        _dropped(7, 33, dtype, p)
    _dropped(3, 40, dtype, 0.3, seed=(1 << 64) - 1, offset=(1 << 64) - 2)
    _dropped(11, 19, dtype, 0.5, residual=False, poison=True)
    _dropped(11, 19, dtype, 0.5, residual=True, poison=True)


def test_dropout_in_place_and_backward():
    """y may be x or the residual; the mask of the gradient is that of the forward pass."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for dtype in (F32, BF16):
        x, r = torch.randn(33, 77, device="cuda", generator=g).to(dtype), torch.randn(33, 77, device="cuda", generator=g).to(dtype)
        ctx = _ctx()
        out = torch.empty_like(x)
        kfac.kfac_dropout(ctx, x, 0.4, 9, 1, out, residual=r)
        inx, inr = x.clone(), r.clone()
        kfac.kfac_dropout(ctx, inx, 0.4, 9, 1, inx, residual=r)
        kfac.kfac_dropout(ctx, x, 0.4, 9, 1, inr, residual=inr)
        assert torch.equal(inx, out) and torch.equal(inr, out)
        grad = torch.empty_like(x)
        kfac.kfac_dropout(ctx, torch.ones_like(x), 0.4, 9, 1, grad)
        t = round(0.4 * 65536)
        f = torch.tensor(65536.0 / (65536.0 - t)).to(dtype).item()
        assert set(grad.unique().tolist()) == {0.0, f}
        # the gradient of sum(y) by differences: y is linear in x where it is kept
        other = torch.empty_like(x)
        kfac.kfac_dropout(ctx, torch.zeros_like(x), 0.4, 9, 1, other)
        assert not bool(other.any())
        kfac.kfac_dropout(ctx, torch.ones_like(x), 0.4, 9, 2, other)     # another offset: another mask
        assert not torch.equal(other, grad)
        ctx.close()


def test_dropout_beyond_32_bit_elements():
    """The counter of an element beyond 2^32: row 2^20 + 1 of rows of 4096 + 8 bf16 elements."""
    rows, cols = (1 << 20) + 2, 4096
    x = torch.ones(rows, cols, dtype=BF16, device="cuda")
    ctx = _ctx()
    kfac.kfac_dropout(ctx, x, 0.5, 11, 0, x)
    last = x[rows - 1].float().cpu().numpy() != 0
    assert np.array_equal(last, T.dropout_keep((rows - 1) * cols, cols, 0.5, 11, 0))
    ctx.close()


@pytest.mark.parametrize("n,num", [(32768, 31), (32769, 31), (32768, 300), (600000, 20), (600000, 70000), (2 ** 21 + 5, 100000)])
def test_segments_of_many_positions(n, num):
    """One workgroup and many tiles, on both sides of the rules that choose between them."""
    ids = np.random.default_rng(n).integers(-1, num, n)
    order, offsets = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(num + 1, dtype=torch.int32, device="cuda")
    ctx = _ctx(kfac.kfac_segments_workspace_bytes(n, num))
    kfac.kfac_segments(ctx, torch.from_numpy(ids).cuda(), num, order, offsets)
    ref_order, ref_offsets = T.segments(ids, num)
    assert np.array_equal(order.cpu().numpy(), ref_order) and np.array_equal(offsets.cpu().numpy(), ref_offsets)
    ctx.close()


def test_embedding_grad_of_unaligned_tables():
    """dW and A_diag that start at any element: the zeros are written around the aligned pieces."""
    rng = np.random.default_rng(8)
    for shift in range(4):
        for n, vocab, dim in ((40, 300, 7), (9000, 500, 3), (0, 5, 3), (1, 1, 1)):
            ids = rng.integers(0, vocab, n)
            g = torch.from_numpy(rng.standard_normal((n, dim))).float().cuda()
            buf, abuf = torch.full((vocab * dim + 8,), 9.0, device="cuda"), torch.full((vocab + 8,), 9.0, device="cuda")
            dW, A = buf[shift:shift + vocab * dim].view(vocab, dim), abuf[shift:shift + vocab]
            ctx = _ctx(kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
            kfac.kfac_embedding_grad(ctx, torch.from_numpy(ids).cuda(), g, 1.0, dW, False, A, 0.0)
            ref, counts, mag = T.embedding_grad(ids, _values(g), 1.0, vocab)
            assert np.all(np.abs(_values(dW) - ref) <= (counts[:, None] + 4) * 2.0 ** -24 * mag)
            assert n == 0 or np.allclose(_values(A), counts / n, rtol=8 * 2.0 ** -24, atol=0)
            for b, size in ((buf, vocab * dim), (abuf, vocab)):
                assert bool((b[:shift] == 9.0).all()) and bool((b[shift + size:] == 9.0).all())
            ctx.close()


@pytest.mark.parametrize("n,share", [(3000, 0.5), (20000, 0.3), (70000, 0.9)])
def test_embedding_grad_of_one_frequent_token(n, share):
    """A token of more parts than one wave adds up, between others, at places that are no whole runs."""
    rng = np.random.default_rng(n)
    vocab, dim = 900, 300
    ids = np.where(rng.random(n) < share, 450, rng.integers(-1, vocab, n))
    g = torch.from_numpy(rng.standard_normal((n, dim))).to(BF16).cuda()
    dW = torch.empty(vocab, dim, device="cuda")
    ctx = _ctx(kfac.kfac_embedding_workspace_bytes(n, vocab, dim))
    kfac.kfac_embedding_grad(ctx, torch.from_numpy(ids).int().cuda(), g, 1.0, dW)
    ref, counts, mag = T.embedding_grad(ids, _values(g), 1.0, vocab)
    assert np.all(np.abs(_values(dW) - ref) <= (counts[:, None] + 4) * 2.0 ** -24 * mag)
    ctx.close()
