"""The float64 implementations of the token and expert layers, pinned: published vectors of the generator, definitions by loops,
gradients by differences, one-hot inputs."""
import numpy as np
import pytest

from oracle import tokens as T


@pytest.mark.parametrize("counter,key,words", [
    # the known answers that come with the generator's publication
    ([0, 0, 0, 0], [0, 0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]),
])
def test_generator(counter, key, words):
    assert T.philox4x32(counter, key) == words


def test_dropout_keeps_the_share_it_says():
    for p in (0.1, 0.5):
        keep = T.dropout_keep(0, 20000, p, 12345, 7)
        # standard deviation sqrt(p (1 - p) / n), five of them
        assert abs(keep.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / 20000)
    assert T.dropout_keep(0, 100, 0.0, 1, 2).all() and not T.dropout_keep(0, 100, 1.0, 1, 2).any()


def test_segments():
    order, offsets = T.segments([3, -1, 0, 3, 9, 0, 2], 4)
    assert order.tolist() == [2, 5, 6, 0, 3, 1, 4] and offsets.tolist() == [0, 2, 2, 3, 5]


def test_embedding_is_a_product_with_one_hot_rows():
    rng = np.random.default_rng(0)
    ids = rng.integers(-1, 7, 40)
    table, g = rng.standard_normal((7, 5)), rng.standard_normal((40, 5))
    hot = np.zeros((40, 7))
    hot[np.nonzero(ids >= 0)[0], ids[ids >= 0]] = 1
    dW, counts, _ = T.embedding_grad(ids, g, 1.5, 7)
    assert np.allclose(T.embedding(ids, table, 1.5), 1.5 * hot @ table, atol=1e-14)
    assert np.allclose(dW, 1.5 * hot.T @ g, atol=1e-13)
    A = hot.T @ hot / 40
    assert np.allclose(A, np.diag(counts / 40), atol=1e-15)      # the factor A is diagonal


@pytest.mark.parametrize("bias", [0, 1])
def test_expert_gradients_by_differences(bias):
    rng = np.random.default_rng(1)
    E, fan, ci, co, tokens = 3, 2, 4, 5, 6
    choice = np.array([0, 2, 2, 0, -1, 0, 2, 2, 0, 0, 2, -1])    # expert 1 has no rows
    x, W, R = rng.standard_normal((tokens, ci)), rng.standard_normal((E, co, ci + bias)), rng.standard_normal((tokens * fan, co))

    def loss(x, W):
        return float((T.expert_forward(choice, x, W, ci, bias, fan)[0] * R).sum())

    dx = T.expert_grad_input(choice, R, W, ci)[0].reshape(tokens, fan, ci).sum(1)
    dW = T.expert_grad_weight(choice, x, R * (choice >= 0)[:, None], E, bias, fan)[0]
    h = 1e-6
    for got, arg in ((dx, 0), (dW, 1)):
        for idx in np.ndindex(got.shape):
            hi, lo = [x.copy(), W.copy()], [x.copy(), W.copy()]
            hi[arg][idx] += h
            lo[arg][idx] -= h
            assert abs((loss(*hi) - loss(*lo)) / (2 * h) - got[idx]) < 1e-7
    assert not dW[1].any()


def test_expert_factors_are_those_of_a_layer_over_the_experts_rows():
    import oracle
    rng = np.random.default_rng(2)
    choice = rng.integers(0, 3, 30)
    x, g = rng.standard_normal((30, 6)).astype(np.float32), rng.standard_normal((30, 4)).astype(np.float32)
    A, _, count = T.expert_factors(choice, x, 3, 1, 1)
    G, _, _ = T.expert_factors(choice, g, 3, 0, 1)
    for e in range(3):
        c = np.nonzero(choice == e)[0]
        L = (len(c), 6, 4, 1, 1, 0, 1, 1, 1)
        Ar, Gr = oracle.kfac_stats(L, x[c].reshape(-1, 6, 1, 1).copy(), g[c].reshape(-1, 4, 1, 1).copy(), 0.0, False, None, None)
        assert count[e] == len(c)
        assert np.allclose(A[e], Ar, atol=1e-12) and np.allclose(G[e], Gr, atol=1e-12)
