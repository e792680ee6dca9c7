"""fp64 oracle of rotary positions and differential attention.

TEST INFRASTRUCTURE ONLY, like the rest of this package; it shares no code with the library.

Rotary positions: pairs of a row's first 2 P elements as complex numbers, times amplitude * exp(i theta) or its conjugate.

Differential attention, one head, over the first `keys` keys:
    A_i = softmax(q_i k_i^T / sqrt(d));  o_i = A_i v;  o = o_1 - lam o_2
    G = dO v^T,  delta_2 = dO . o2,  delta_1 = dO . o + lam delta_2   (from the outputs that the caller holds)
    S_1 = A_1 o (G - delta_1),  S_2 = -lam A_2 o (G - delta_2)
    dv = (A_1 - lam A_2)^T dO,  dq_i = S_i k_i / sqrt(d),  dk_i = S_i^T q_i / sqrt(d),  dlam = -sum delta_2

Beside each result stands how far a computation may be from it that rounds probabilities, S and the results to bf16
(half a step, 2^-8 of the value) and does everything else in fp32 (2^-24 for each rounding behind a score, an inner
product or an exponent), propagated through the formulas with absolute values.
"""

from __future__ import annotations

import numpy as np

__all__ = ["rope", "rope_tolerance", "forward", "backward"]

HALF_BF16 = 2.0 ** -8
HALF_F32 = 2.0 ** -24
TINY = 1e-30  # below it bf16 and fp32 lose bits to the exponent's range


def rope(x, positions, freq, axis=None, amplitude=1.0, layout="interleaved", inverse=False):
    """x [B,H,T,D]; positions [T] or [B,T], with a last dimension of coordinates where axis is given."""
    x, P = np.asarray(x, dtype=np.float64), len(freq)
    p = np.asarray(positions, dtype=np.float64)
    p = p[..., None] * np.ones(P) if axis is None else p[..., np.asarray(axis)]
    turn = amplitude * np.exp((-1j if inverse else 1j) * p * np.asarray(freq, dtype=np.float64))
    turn = turn if turn.ndim == 2 else turn[:, None]
    y = x.copy()
    a, b = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "interleaved" else (slice(0, P), slice(P, 2 * P))
    z = (x[..., a] + 1j * x[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y


def rope_tolerance(x, y, P, half_step, amplitude=1.0, layout="interleaved", largest=0.0):
    """A rounding of the result, and 6 roundings of 32 bits against the pair's elements: the angle is within a quarter
    turn's part of 2.5 of them, its cosine one more, the amplitude, the products and their sum one each.  largest: the
    largest angle, which is itself a product in 64 bits: one rounding of it (2^-53) above, three in a computation that
    counts turns (1 / 2 pi, its product with the frequency, and that with the position)."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    a, b = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if layout == "interleaved" else (slice(0, P), slice(P, 2 * P))
    tol = half_step * np.abs(y)
    pair = (6 * HALF_F32 + 4 * 2.0 ** -53 * largest) * abs(amplitude) * (x[..., a] + x[..., b])
    tol[..., a] += pair
    tol[..., b] += pair
    tol[..., 2 * P:] = 0.0
    # below the smallest normal number of an 8-bit or 5-bit exponent half a step is a fixed amount
    return tol + (2.0 ** -25 if half_step == 2.0 ** -11 else TINY)


def _scores(q, k, d, keys, x_tol=False):
    s = q @ k[:keys].T / np.sqrt(d)
    if not x_tol:
        return s
    # d products and sums, the scale and the subtraction behind an exponent
    return s, (d + 8) * HALF_F32 * (np.abs(q) @ np.abs(k[:keys]).T / np.sqrt(d) + np.abs(s).max(initial=0.0) + 1.0)


def forward(q, k, v, lam, keys, pieces=1, waves=1):
    """q, k: two maps [T,d] each; v [Tk, 2d].  (o, o2, m, l) with m, l [2,T], and their tolerances in the same order.
    pieces: the numbers of bf16 that a probability is taken in, each the rounding of what those before it leave.  waves: that
    share the keys 32 by 32, each with a sum of its own."""
    d, out, tol, ms, ls, mt, lt = q[0].shape[1], [], [], [], [], [], []
    adds = keys if waves == 1 else keys // waves + 32 + waves
    for i in range(2):
        s, e_s = _scores(q[i], k[i], d, keys, True)
        m = s.max(1, initial=-np.inf)
        e = np.exp(s - np.where(np.isfinite(m), m, 0.0)[:, None])
        l = e.sum(1)
        A = e / np.where(l > 0, l, 1.0)[:, None]
        out.append(A @ v[:keys])
        # probabilities rounded to bf16 against the running max, their sum not; both off by the scores' errors
        rel = HALF_BF16 ** pieces + 2 * e_s + pieces * adds * HALF_F32
        tol.append((A * rel) @ np.abs(v[:keys]))
        ms.append(m)
        ls.append(l)
        mt.append(e_s.max(1, initial=0.0) + HALF_F32 * np.where(np.isfinite(m), np.abs(m), 0.0))
        lt.append(l * (2 * e_s.max(1, initial=0.0) + (keys + 8) * HALF_F32))
    o = out[0] - lam * out[1]
    t2 = tol[1] + HALF_BF16 * np.abs(out[1])
    t = tol[0] + abs(lam) * tol[1] + HALF_BF16 * np.abs(o) + 4 * HALF_F32 * (np.abs(out[0]) + abs(lam * out[1]))
    return (o, out[1], np.stack(ms), np.stack(ls)), (t + TINY, t2 + TINY, np.stack(mt) + TINY, np.stack(lt) + TINY)


def backward(q, k, v, o, o2, m, l, d_o, lam, keys):
    """(dq [2,Tq,d], dk [2,Tk,d], dv, dlam) and their tolerances."""
    d, v0 = q[0].shape[1], v[:keys]
    delta2 = (d_o * o2).sum(1)
    deltas = (d_o * o).sum(1) + lam * delta2, delta2
    gains = 1.0, -lam
    G = d_o @ v0.T
    wide = 2 * d + 8
    e_G = wide * HALF_F32 * (np.abs(d_o) @ np.abs(v0).T + (np.abs(d_o) * (np.abs(o) + 2 * abs(lam) * np.abs(o2) + np.abs(o2))).sum(1)[:, None])
    dq, dk = np.zeros((2,) + q[0].shape), np.zeros((2,) + k[0].shape)
    tq, tk = np.zeros_like(dq), np.zeros_like(dk)
    A, e_A = [], []
    for i in range(2):
        s, e_s = _scores(q[i], k[i], d, keys, True)
        a = np.exp(s - np.where(l[i] > 0, m[i], 0.0)[:, None]) / np.where(l[i] > 0, l[i], 1.0)[:, None]
        rel = 2 * e_s + 4 * HALF_F32 * (np.abs(np.where(l[i] > 0, m[i], 0.0)) + np.abs(np.log(np.where(l[i] > 0, l[i], 1.0))) + 2)[:, None]
        A.append(a)
        e_A.append(a * rel)
        S = a * (G - deltas[i][:, None]) * gains[i]
        e_S = (HALF_BF16 + rel) * np.abs(S) + a * e_G * abs(gains[i])
        f = 1 / np.sqrt(d)
        dq[i], dk[i, :keys] = S @ k[i][:keys] * f, S.T @ q[i] * f
        more = (q[0].shape[0] + keys) * HALF_F32
        tq[i] = (e_S + more * np.abs(S)) @ np.abs(k[i][:keys]) * f + (HALF_BF16 + 8 * HALF_F32) * np.abs(dq[i])
        tk[i, :keys] = (e_S + more * np.abs(S)).T @ np.abs(q[i]) * f + (HALF_BF16 + 8 * HALF_F32) * np.abs(dk[i, :keys])
    W = A[0] - lam * A[1]
    dv, tv = np.zeros_like(v), np.zeros_like(v)
    dv[:keys] = W.T @ d_o
    e_W = HALF_BF16 * np.abs(W) + e_A[0] + abs(lam) * e_A[1] + len(d_o) * HALF_F32 * (A[0] + abs(lam) * A[1])
    tv[:keys] = e_W.T @ np.abs(d_o) + HALF_BF16 * np.abs(dv[:keys])
    dlam = -delta2.sum()
    tl = (wide * np.abs(d_o * o2).sum() + abs(dlam)) * HALF_F32
    return (dq, dk, dv, dlam), (tq + TINY, tk + TINY, tv + TINY, tl + TINY)
