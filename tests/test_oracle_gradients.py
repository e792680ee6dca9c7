"""The gradient oracle against differences of the forward definitions (CPU)."""

import numpy as np
import pytest

from oracle import attention as oa
from oracle import gradients as og


def _forward(q, k, v, kept, w):
    s = np.where(kept, q @ k.T / np.sqrt(q.shape[1]), -np.inf)
    m = s.max(1)
    e = np.exp(s - m[:, None])
    l = e.sum(1)
    return (e @ v) / l[:, None] * w[:, None], m, l


@pytest.mark.parametrize("masked", [False, True])
def test_attention_gradients_are_differences(masked):
    rng = np.random.default_rng(5)
    T, d = 9, 6
    q, k, v, d_o = (rng.standard_normal((T, d)) for _ in range(4))
    w = rng.uniform(0.1, 1.0, T) if masked else np.ones(T)
    kept = np.ones((T, T), dtype=bool)
    if masked:
        kept = og.token_mask(np.array([0, 2, 3, 5]), np.array([0, 2, 1, 0, 2]), 3, T)
    out, m, l = _forward(q, k, v, kept, w)
    got = og.head_backward(q, k, v, out / w[:, None], m, l, d_o, kept, w)
    h = 1e-5
    for x, grad in zip((q, k, v), got):
        num = np.empty_like(x)
        for i in np.ndindex(*x.shape):
            was = x[i]
            x[i] = was + h
            up = (_forward(q, k, v, kept, w)[0] * d_o).sum()
            x[i] = was - h
            down = (_forward(q, k, v, kept, w)[0] * d_o).sum()
            x[i] = was
            num[i] = (up - down) / (2 * h)
        # second-order differences: h^2 times a third derivative of order one, and 1e-16 / h of rounding
        assert np.abs(num - grad).max() <= 1e-8
    # the gradient for the factor w is delta
    num = [((_forward(q, k, v, kept, w + h * np.eye(T)[i])[0] - _forward(q, k, v, kept, w - h * np.eye(T)[i])[0])
            * d_o).sum() / (2 * h) for i in range(T)]
    assert np.abs(np.array(num) - got[3]).max() <= 1e-8


def test_dense_gradients_use_the_forward_oracle():
    rng = np.random.default_rng(6)
    q, k, v, d_o = (rng.standard_normal((1, 2, 40, 64)) for _ in range(4))
    o, m, l = oa.full_attention(q, k, v)
    for h in range(2):
        dq, dk, dv, delta = og.head_backward(q[0, h], k[0, h], v[0, h], o[0, h], m[0, h], l[0, h], d_o[0, h])
        # rows of dS sum to zero, so dQ . Q and dK . K have equal sums; columns of P sum to dV's weights
        assert abs((dq * q[0, h]).sum() - (dk * k[0, h]).sum()) < 1e-10
        assert np.abs(delta - (d_o[0, h] * o[0, h]).sum(1)).max() == 0
        assert np.abs(dv.sum(0) - d_o[0, h].sum(0)).max() < 1e-12


def test_tolerances_hold_for_rounded_products():
    """A computation in fp32 with P, dS and results rounded to bf16 stays inside the bounds, one with dS kept to
    six bits does not."""
    rng = np.random.default_rng(7)
    T, d = 64, 64

    def bf16(x, bits=8):
        mant, e = np.frexp(x)
        return np.ldexp(np.round(mant * 2 ** bits) / 2 ** bits, e)

    q, k, v, d_o = (bf16(rng.standard_normal((T, d))) for _ in range(4))
    kept = np.ones((T, T), dtype=bool)
    o, m, l = _forward(q, k, v, kept, np.ones(T))
    o = bf16(o)
    ref, tol = og.head_backward(q, k, v, o, m, l, d_o), og.head_tolerances(q, k, v, o, m, l, d_o)
    p = np.exp(q @ k.T / 8 - m[:, None]) / l[:, None]
    ds = p * (d_o @ v.T - (d_o * o).sum(1)[:, None])
    dq = bf16(bf16(ds) @ k / 8)
    assert (np.abs(dq - ref[0]) <= tol[0]).all()
    assert (np.abs(bf16(bf16(p).T @ d_o) - ref[2]) <= tol[2]).all()
    assert not (np.abs(bf16(bf16(ds, 4) @ k / 8) - ref[0]) <= tol[0]).all()


def test_layer_norm_gradients_are_differences():
    rng = np.random.default_rng(8)
    x, w, b, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    _, mean, rstd = og.layer_norm(x, w, b, 1e-3)
    dx, dw, db = og.layer_norm_backward(dy, x, mean, rstd, w)
    h = 1e-5
    for t, grad in ((x, dx), (w, dw.sum(0)), (b, db.sum(0))):
        for i in np.ndindex(*t.shape):
            was = t[i]
            t[i] = was + h
            up = (og.layer_norm(x, w, b, 1e-3)[0] * dy).sum()
            t[i] = was - h
            down = (og.layer_norm(x, w, b, 1e-3)[0] * dy).sum()
            t[i] = was
            assert abs((up - down) / (2 * h) - grad[i]) <= 1e-7
