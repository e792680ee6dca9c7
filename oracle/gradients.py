"""fp64 oracle of the training operators: gradients of attention, and the layer norm with its gradients.

TEST INFRASTRUCTURE ONLY, like the rest of this package; it shares no code with the library.

Attention (one head, kept pairs given as a boolean T x T matrix, all true for dense attention), from the output o
and the row statistics m, l of the forward call and a factor w per query row:
    P_ij  = w_i exp(q_i . k_j / sqrt(d) - m_i) / l_i          for kept pairs, else 0
    delta_i = dO_i . o_i
    dV = P^T dO,  dS = P o (dO V^T - delta),  dQ = dS K / sqrt(d),  dK = dS^T Q / sqrt(d)

Beside each gradient stands `tol`, how far a computation may be from it that rounds P, dS and the result to bf16
(half a step, 2^-8 of the value) and does everything else in fp32 (2^-24 for each of the at most D + 8 roundings
behind a score or an inner product): the bound is propagated through the formulas with absolute values.
"""

from __future__ import annotations

import numpy as np

__all__ = ["head_backward", "head_tolerances", "token_mask", "layer_norm", "layer_norm_backward"]

HALF_BF16 = 2.0 ** -8
HALF_F32 = 2.0 ** -24
TINY = 1e-30  # below it bf16 and fp32 lose bits to the exponent's range


def token_mask(row_ptr, col_idx, block, T):
    """Boolean T x T of the kept pairs of one block CSR."""
    n = -(-T // block)
    blocks = np.zeros((n, n), dtype=bool)
    for i in range(n):
        blocks[i, np.asarray(col_idx[row_ptr[i]:row_ptr[i + 1]], dtype=np.int64)] = True
    at = np.arange(T) // block
    return blocks[at][:, at]


def _probabilities(q, k, m, l, kept, w):
    s = (q @ k.T) / np.sqrt(q.shape[1])
    with np.errstate(over="ignore"):
        return np.where(kept, np.exp(np.where(kept, s - m[:, None], 0.0)) / l[:, None], 0.0) * w[:, None]


def head_backward(q, k, v, o, m, l, d_o, kept=None, w=None):
    """dQ, dK, dV and delta of one head (float64 [T, d] and [T])."""
    T, d = q.shape
    kept = np.ones((T, T), dtype=bool) if kept is None else kept
    p = _probabilities(q, k, m, l, kept, np.ones(T) if w is None else w)
    delta = (d_o * o).sum(1)
    ds = p * (d_o @ v.T - delta[:, None])
    return ds @ k / np.sqrt(d), ds.T @ q / np.sqrt(d), p.T @ d_o, delta


def head_tolerances(q, k, v, o, m, l, d_o, kept=None, w=None):
    """Bounds on the error of dQ, dK, dV and delta, element by element (see above)."""
    T, d = q.shape
    kept = np.ones((T, T), dtype=bool) if kept is None else kept
    p = _probabilities(q, k, m, l, kept, np.ones(T) if w is None else w)
    r = (d + 8) * HALF_F32
    # the exponent in units of log2: its own roundings, those of the row's logarithm, the exp2 itself
    size = np.abs(q) @ np.abs(k).T / np.sqrt(d) * np.log2(np.e)
    log = (np.abs(m) * np.log2(np.e) + np.abs(np.log2(l)) + (0 if w is None else np.abs(np.log2(np.maximum(w, TINY)))))
    e_p = p * (r * size + 4 * HALF_F32 * (log[:, None] + size) + 4 * HALF_F32)
    delta = (d_o * o).sum(1)
    e_delta = r * (np.abs(d_o) * np.abs(o)).sum(1)
    dp = d_o @ v.T - delta[:, None]
    e_dp = r * (np.abs(d_o) @ np.abs(v).T) + e_delta[:, None] + 2 * HALF_F32 * np.abs(dp)
    ds = np.abs(p * dp)
    e_ds = e_p * np.abs(dp) + (p + e_p) * e_dp
    e_ds += HALF_BF16 * (ds + e_ds)
    e_p = e_p + HALF_BF16 * (p + e_p)
    c = 1 / np.sqrt(d)
    out = []
    for ref, size, err in ((np.abs((p * dp) @ k), ds @ np.abs(k), e_ds @ np.abs(k)),
                           (np.abs((p * dp).T @ q), ds.T @ np.abs(q), e_ds.T @ np.abs(q))):
        err = err + (T + 8) * HALF_F32 * (size + err)  # the sum over tokens
        out.append(c * (err + HALF_BF16 * (ref + err)) + TINY)
    size, err = p.T @ np.abs(d_o), e_p.T @ np.abs(d_o)
    err = err + (T + 8) * HALF_F32 * (size + err)
    out.append(err + HALF_BF16 * (np.abs(p.T @ d_o) + err) + TINY)
    return out[0], out[1], out[2], e_delta + TINY


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """y, mean, rstd of rows [.., W]; weight and bias broadcast against x."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[..., None]) * rstd[..., None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def layer_norm_backward(d_y, x, mean, rstd, weight=None):
    """dx, and for each row its terms of d_weight (dy xh) and d_bias (dy), to be summed over the rows of a set."""
    d_y, x = np.asarray(d_y, dtype=np.float64), np.asarray(x, dtype=np.float64)
    xh = (x - mean[..., None]) * rstd[..., None]
    g = d_y if weight is None else d_y * weight
    dx = rstd[..., None] * (g - g.mean(-1, keepdims=True) - xh * (g * xh).mean(-1, keepdims=True))
    return dx, d_y * xh, d_y
