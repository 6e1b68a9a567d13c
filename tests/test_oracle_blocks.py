"""The float64 implementations around the products of experts, pinned: definitions by loops, gradients by differences, published
values of the 8-bit format."""
import numpy as np
import pytest

from oracle import blocks as B

INF = np.inf


def test_scores():
    l = np.array([[0.0, np.log(3.0), -INF], [-INF, -INF, -INF]])
    assert np.allclose(B.scores(l, False), [[0.25, 0.75, 0.0], [0, 0, 0]], atol=1e-16)
    assert np.allclose(B.scores(np.array([[0.0, np.log(3.0), -INF, 800.0, -800.0]]), True), [[0.5, 0.75, 0.0, 1.0, 0.0]], atol=1e-16)


def test_route_takes_the_best_and_the_lower_number():
    l = np.array([[1.0, 3.0, 3.0, 0.0], [-INF, 2.0, -INF, -INF], [-INF] * 4, [np.nan, 1, 2, 3]])
    c, g = B.route(l, None, 2)
    assert c.tolist() == [[1, 2], [1, -1], [-1, -1], [-1, -1]]
    assert np.allclose(g[:3], [[0.5, 0.5], [1, 0], [0, 0]]) and np.isnan(g[3]).all()
    bias = np.array([10.0, 0, 0, -INF])
    c, g = B.route(l[:1], bias, 3, sigmoid=True, renormalise=False, scale=2.0)
    assert c.tolist() == [[0, 1, 2]] and np.allclose(g, 2 * B.scores(l[:1], True)[:, [0, 1, 2]])


def test_route_groups():
    # best single expert in group 2, best pair in group 0
    l = np.array([[2.0, 2.0, 0.0, 0.0, 2.5, -9.0, 1.0, 1.0]])
    assert B.route(l, None, 2, groups=4, top_groups=1)[0].tolist() == [[4, 5]]
    assert B.route(l, None, 2, groups=4, top_groups=1, group_best=2, sigmoid=True)[0].tolist() == [[0, 1]]
    assert B.route(l, None, 3, groups=4, top_groups=2)[0].tolist() == [[4, 0, 1]]


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient_by_differences(sigmoid, renormalise):
    rng = np.random.default_rng(3)
    l, d = rng.standard_normal((6, 9)), rng.standard_normal((6, 3))
    l[2, 4], l[3] = -INF, -INF
    options = dict(sigmoid=sigmoid, renormalise=renormalise, scale=1.7)
    c, _ = B.route(l, None, 3, **options)
    got, mag = B.route_grad(l, c, d, **options)
    assert (np.abs(got) <= mag * (1 + 1e-12)).all() and not got[3].any()

    def loss(x):
        s = B.scores(x, sigmoid)
        total = 0.0
        for t in range(6):
            j = c[t] >= 0
            g = s[t, c[t][j]]
            if j.any():
                total += (1.7 * (g / g.sum() if renormalise else g) * d[t][j]).sum()
        return total
    for t in range(6):
        for e in range(9):
            if np.isfinite(l[t, e]):
                up, down = l.copy(), l.copy()
                up[t, e] += 1e-5
                down[t, e] -= 1e-5
                assert abs((loss(up) - loss(down)) / 2e-5 - got[t, e]) < 1e-8   # (third derivatives below 10, rounding 1e-16 / 1e-5)


def test_weights_of_tiny_sigmoids():
    w = B.weights(np.array([-900.0, -901.0, 0.0]), np.array([0, 1]), True)
    assert np.allclose(w, [1 / (1 + np.exp(-1)), np.exp(-1) / (1 + np.exp(-1))], atol=1e-15)


def test_combine_and_its_gradients():
    rng = np.random.default_rng(4)
    y, g, r, d = rng.standard_normal((6, 5)), rng.standard_normal(6), rng.standard_normal((3, 5)), rng.standard_normal((3, 5))
    out, mag = B.combine(y, g, 2, r)
    for t in range(3):
        assert np.allclose(out[t], r[t] + g[2 * t] * y[2 * t] + g[2 * t + 1] * y[2 * t + 1])
    assert (np.abs(out) <= mag + 1e-15).all()
    dy, dg, _ = B.combine_grad(y, g, 2, d)
    loss = lambda y_, g_: (B.combine(y_, g_, 2, r)[0] * d).sum()  # noqa: E731
    for i in range(6):
        e = np.zeros(6)
        e[i] = 1.0
        assert abs(loss(y, g + e) - loss(y, g) - dg[i]) < 1e-12       # linear
        for c in range(5):
            z = np.zeros((6, 5))
            z[i, c] = 1.0
            assert abs(loss(y + z, g) - loss(y, g) - dy[i, c]) < 1e-12


def test_e4m3():
    v = B.e4m3_values()
    # the published corners of the format: largest, smallest normal, largest and smallest subnormal
    assert v[0x7E] == 448 and v[0x08] == 2.0 ** -6 and v[0x07] == 0.875 * 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[0xB8] == -1.0
    fine = np.array([b for b in range(256) if b & 0x7F != 0x7F], dtype=np.uint8)
    assert np.array_equal(B.to_e4m3(v[fine]), fine)
    ties = np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0001, -17.0])    # between 16 and 18, 18 and 20, 0 and 2^-9, ...
    assert v[B.to_e4m3(ties)].tolist() == [16.0, 20.0, 0.0, 2.0 ** -8, 18.0, -16.0]


def test_keep():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 70)) * 10.0 ** rng.integers(-30, 30, (4, 70))
    x[0, :32] = 0.0
    x[1, 3], x[1, 40] = INF, -np.nan
    x[2, 0] = 448.0
    x[2, 1:32] = 1.0
    q, s = B.keep(x)
    v = B.restore(q, s)
    assert s[0, 0] == 10 and s[2, 0] == 127 and v[2, 0] == 448 and (v[2, 1:32] == 1).all()
    assert np.isnan(v[1, 3]) and np.isnan(v[1, 40]) and np.isfinite(np.delete(v, 0, 1)[0]).all()
    fine = np.isfinite(x)
    power = np.repeat(2.0 ** (s.astype(float) - 127), 32, 1)[:, :70]
    assert (np.abs(v - x)[fine] <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * power)[fine]).all()
    high = np.array([[np.where(fine, np.abs(x), 0)[r, 32 * b:32 * b + 32].max() for b in range(3)] for r in range(4)])
    power = 2.0 ** (s.astype(float) - 127)
    assert (high <= 448 * power).all() and ((high > 224 * power) | (s == 10)).all()


def test_rms_norm_gradient_by_differences():
    rng = np.random.default_rng(6)
    h, gamma, dy, ds = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    y, r = B.rms_norm(h, gamma, 1e-3)
    assert np.allclose(y[1], gamma * h[1] / np.sqrt(np.mean(h[1] ** 2) + 1e-3))
    dh, mag, dg, gmag, F = B.rms_norm_grad(dy, h, gamma, 1e-3, ds)
    assert (np.abs(dh) <= mag + 1e-14).all() and (np.abs(dg) <= gmag + 1e-14).all()
    loss = lambda h_, g_: (B.rms_norm(h_, g_, 1e-3)[0] * dy).sum() + (h_ * ds).sum()  # noqa: E731
    for t in range(3):
        for c in range(7):
            z = np.zeros((3, 7))
            z[t, c] = 1e-5
            assert abs((loss(h + z, gamma) - loss(h - z, gamma)) / 2e-5 - dh[t, c]) < 1e-7
    for c in range(7):
        z = np.zeros(7)
        z[c] = 1.0
        assert abs(loss(h, gamma + z) - loss(h, gamma) - dg[c]) < 1e-12
    per_token = dy * h * r
    assert np.allclose(F, np.mean(per_token ** 2, 0)) and np.allclose(dg, per_token.sum(0))
