"""The oracle of rotary positions and differential attention against differences and plain definitions (CPU)."""

import numpy as np
import pytest

from oracle import heads as oh


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rotation_keeps_lengths_and_inner_products_go_by_distance(layout):
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 1, 1, 1, 16))
    freq = 100.0 ** (-np.arange(6) / 6)
    turned = [oh.rope(x, [p], freq, layout=layout) for p in (3, 10)], [oh.rope(y, [p], freq, layout=layout) for p in (5, 12)]
    for a in turned[0]:
        assert abs((a ** 2).sum() - (x ** 2).sum()) < 1e-12
        assert np.array_equal(a[..., 12:], x[..., 12:])
    assert abs((turned[0][0] * turned[1][0]).sum() - (turned[0][1] * turned[1][1]).sum()) < 1e-12
    back = oh.rope(turned[0][0], [3], freq, layout=layout, inverse=True)
    assert np.abs(back - x).max() < 1e-14
    # a pair by hand
    c, s = np.cos(3 * freq[1]), np.sin(3 * freq[1])
    i, j = (2, 3) if layout == "interleaved" else (1, 7)
    assert np.abs(turned[0][0][0, 0, 0, [i, j]] - [x[0, 0, 0, i] * c - x[0, 0, 0, j] * s, x[0, 0, 0, i] * s + x[0, 0, 0, j] * c]).max() < 1e-14


def test_rotation_takes_each_pairs_axis_and_each_samples_positions():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((2, 3, 4, 8))
    freq, pos = [1.0, 0.5, 1.0, 0.1], rng.integers(0, 50, (2, 4, 2))
    y = oh.rope(x, pos, freq, axis=[0, 0, 1, 1])
    for b in range(2):
        for p in range(4):
            one = oh.rope(x[b:b + 1, :, :, 2 * p:2 * p + 2], pos[b, :, p // 2], freq[p:p + 1])
            assert np.abs(one[0] - y[b, :, :, 2 * p:2 * p + 2]).max() < 1e-14


@pytest.mark.parametrize("keys", [7, 4, 0])
def test_gradients_are_differences(keys):
    rng = np.random.default_rng(3)
    q, k, v, d_o = rng.standard_normal((2, 5, 6)), rng.standard_normal((2, 7, 6)), rng.standard_normal((7, 12)), rng.standard_normal((5, 12))
    lam = np.array([0.7])
    value = lambda: (oh.forward(q, k, v, lam[0], keys)[0][0] * d_o).sum()  # noqa: E731
    (o, o2, m, l), _ = oh.forward(q, k, v, lam[0], keys)
    got, tol = oh.backward(q, k, v, o, o2, m, l, d_o, lam[0], keys)
    h = 1e-5
    for x, grad in zip((q, k, v, lam), (*got[:3], np.array([got[3]]))):
        for i in np.ndindex(*x.shape):
            was = x[i]
            x[i] = was + h
            up = value()
            x[i] = was - h
            down = value()
            x[i] = was
            # second-order differences: h^2 times a third derivative of order one, and 1e-16 / h of rounding
            assert abs((up - down) / (2 * h) - grad[i]) <= 1e-8, i
    assert all(np.isfinite(t).all() for t in tol)
    if keys == 0:
        assert np.all(o == 0) and np.all(m == -np.inf) and np.all(l == 0) and all(np.all(g == 0) for g in got)


def test_forward_is_two_softmax_maps():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((2, 3, 4)), rng.standard_normal((2, 6, 4)), rng.standard_normal((6, 8))
    (o, o2, m, l), _ = oh.forward(q, k, v, 0.3, 5)
    maps = []
    for i in range(2):
        e = np.exp(q[i] @ k[i][:5].T / 2)
        maps.append(e / e.sum(1, keepdims=True))
        assert np.abs(np.log(l[i]) + m[i] - np.log(e.sum(1))).max() < 1e-12
    assert np.abs(o - (maps[0] - 0.3 * maps[1]) @ v[:5]).max() < 1e-14
    assert np.abs(o2 - maps[1] @ v[:5]).max() < 1e-14
