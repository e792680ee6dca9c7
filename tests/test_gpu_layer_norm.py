"""Layer norm and its gradients against the 64-bit oracle.

Bounds, element by element: a sum of n terms in fp32 whose order is a lane's share, then lanes, waves and workgroups
has at most DEPTH additions behind any term, each off by half a step (2^-24) of what it adds up to, so its error is at
most DEPTH 2^-24 times the sum of magnitudes; everything else has a few roundings (counted below), and the result's
type half a step more."""

import ctypes

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import gradients as og

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROW_DEPTH = 64    # a lane's 32 elements, 6 steps over lanes, 16 waves, and room
COL_DEPTH = 256   # a lane's rows, 3 steps, 4 waves, 16 partial sums a slice, 64 slices, and room
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": U}
# what a result loses where its type runs out of exponent
TINY = {"bf16": 1e-38, "fp16": 2.0 ** -25, "fp32": 1e-38}


def _types():
    import torch

    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _np(t):
    return t.double().cpu().numpy()


def _tensor(shape, dtype, seed, scale=1.0, shift=0.0):
    import torch

    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(_types()[dtype]).cuda()


def _inside(got, ref, tol, what):
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    err = np.abs(got - ref)
    assert (err <= tol).all(), f"{what}: off {err.max():.3e}, worst {np.max(err / tol):.2f} of what is allowed"


def _broadcast(w, x):
    w = _np(w)
    return w if w.ndim == 1 else w.reshape(w.shape[0], *[1] * (x.ndim - 2), -1)


def _check_forward(x, weight, bias, eps, out, dtype):
    y, mean, rstd = out
    X = _np(x)
    w = 1.0 if weight is None else _broadcast(weight, X)
    b = 0.0 if bias is None else _broadcast(bias, X)
    ref, m, r = og.layer_norm(X, w, b, eps)
    e_mean = ROW_DEPTH * U * np.abs(X).mean(-1) + U * np.abs(m)
    d = np.abs(X - m[..., None])
    e_d = e_mean[..., None] + U * d
    var = (d ** 2).mean(-1)
    e_var = (2 * d * e_d + e_d ** 2).mean(-1) + ROW_DEPTH * U * var + 2 * U * (var + eps)
    rel_r = 0.5 * e_var / np.maximum(var + eps - e_var, 1e-300) + 4 * U
    _inside(_np(mean), m, e_mean + 1e-38, "mean")
    _inside(_np(rstd), r, rel_r * r + 1e-38, "rstd")
    xh = d * r[..., None]
    e_y = np.abs(w) * (e_d * r[..., None] + xh * rel_r[..., None] + 2 * U * xh) * (1 + 1e-3) + 2 * U * (np.abs(w) * xh + np.abs(b))
    _inside(_np(y), ref, e_y + HALF[dtype] * (np.abs(ref) + e_y) + TINY[dtype], "y")


def _check_backward(dy, x, mean, rstd, weight, out, dtype, bias=True):
    dx, dw, db = out
    X, G, M, R = _np(x), _np(dy), _np(mean), _np(rstd)
    w = 1.0 if weight is None else _broadcast(weight, X)
    ref, tw, tb = og.layer_norm_backward(G, X, M, R, w)
    xh = np.abs((X - M[..., None]) * R[..., None])
    e_xh = 3 * U * xh
    g = np.abs(G * w)
    s1, s2 = np.abs((G * w).mean(-1, keepdims=True)), np.abs((G * w * (X - M[..., None]) * R[..., None]).mean(-1, keepdims=True))
    e_s1 = (ROW_DEPTH + 2) * U * g.mean(-1, keepdims=True)
    e_s2 = (ROW_DEPTH + 2) * U * (g * xh).mean(-1, keepdims=True) + (g * e_xh).mean(-1, keepdims=True)
    e_dx = R[..., None] * (e_s1 + e_xh * s2 + xh * e_s2 + 5 * U * (g + s1 + xh * s2)) * (1 + 1e-3)
    _inside(_np(dx), ref, e_dx + HALF[dtype] * (np.abs(ref) + e_dx) + TINY[dtype], "dx")
    if weight is None:
        assert dw is None and db is None
        return
    over = tuple(range(1 if weight.dim() == 2 else 0, X.ndim - 1))
    _inside(_np(dw), tw.sum(over), COL_DEPTH * U * np.abs(tw).sum(over) + (np.abs(G) * e_xh).sum(over) + 1e-37, "d_weight")
    if bias:
        _inside(_np(db), tb.sum(over), COL_DEPTH * U * np.abs(tb).sum(over) + 1e-37, "d_bias")
    else:
        assert db is None


def _both(x, dy, weight, bias, dtype, eps=1e-5, out=None, dx=None):
    fwd = rt.layer_norm(x, weight, bias, eps=eps, stats=True, out=out)
    _check_forward(x, weight, bias, eps, fwd, dtype)
    _check_backward(dy, x, fwd[1], fwd[2], weight, rt.layer_norm_backward(dy, x, fwd[1], fwd[2], weight, out=dx), dtype)


# widths on both sides of each choice of lanes and chunks, whole 8-element pieces and odd ones
WIDTHS = [1, 2, 7, 8, 16, 17, 63, 64, 65, 72, 128, 129, 136, 256, 257, 264, 512, 513, 520, 1000, 1024, 1032, 1152, 1536,
          1544, 1920, 2048, 2049, 2056, 4096, 4104, 5001, 8192, 8193, 8200, 16383, 16384]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("W", WIDTHS)
def test_widths(gpu, W, dtype):
    print(f"[layer norm] W={W} {dtype}", flush=True)
    rows = 37 if W < 4000 else 5
    x, dy = _tensor((2, rows, W), dtype, W, 1.5, 0.3), _tensor((2, rows, W), dtype, W + 1)
    wt = dtype if W % 2 else "fp32"
    _both(x, dy, _tensor((W,), wt, 2, 0.2, 1.0), _tensor((W,), wt, 3, 0.2), dtype)


@pytest.mark.parametrize("rows", [1, 2, 3, 31, 33, 127, 129, 1025, 5000, 70001])
@pytest.mark.parametrize("W", [24, 64, 65, 1152])
def test_row_counts(gpu, rows, W):
    if rows * W > 10_000_000:
        pytest.skip("the oracle would take long")
    x, dy = _tensor((rows, W), "bf16", rows, 1.5, 0.3), _tensor((rows, W), "bf16", rows + 1)
    _both(x, dy, _tensor((W,), "fp32", 2, 0.2, 1.0), _tensor((W,), "fp32", 3, 0.2), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,N,W", [(1, 5, 64), (3, 300, 72), (2, 700, 1152), (5, 1, 33), (40, 7, 16), (1100, 3, 64)])
def test_weights_for_each_sample(gpu, B, N, W, dtype):
    x, dy = _tensor((B, N, W), dtype, 1, 1.5, 0.3), _tensor((B, N, W), dtype, 2)
    _both(x, dy, _tensor((B, W), "fp32", 3, 0.2, 1.0), _tensor((B, W), "fp32", 4, 0.2), dtype)


@pytest.mark.parametrize("D", [64, 72, 71])
def test_heads_of_a_packed_projection(gpu, D):
    import torch

    B, N, H = 2, 77, 5
    packed = _tensor((B, N, 3, H, D), "bf16", 5, 1.5, 0.3)
    grad = torch.full_like(packed, 7.0)
    w, b = _tensor((D,), "fp32", 6, 0.2, 1.0), _tensor((D,), "fp32", 7, 0.2)
    for i in range(2):
        x, dx = (t[:, :, i].transpose(1, 2) for t in (packed, grad))
        _both(x, _tensor((B, H, N, D), "bf16", 8 + i), w, b, "bf16", dx=dx)
    assert (grad[:, :, 2] == 7.0).all()  # what lies between the rows stays as it was
    # and written out in a layout of its own
    y = torch.zeros((N, H, B, D), dtype=torch.bfloat16, device="cuda").permute(2, 1, 0, 3)
    _both(packed[:, :, 0].transpose(1, 2), _tensor((B, H, N, D), "bf16", 9), w, b, "bf16", out=y)


def test_strides_of_zero_and_unaligned_rows(gpu):
    import torch

    # one gradient row for all rows, rows that start 2 bytes off, a row stride that is no multiple of 16 bytes
    buf = _tensor((40 * 131 + 1,), "bf16", 10, 1.5, 0.3)
    x = buf[1:].as_strided((40, 128), (131, 1), 1)
    dy = _tensor((1, 128), "bf16", 11).expand(40, 128)
    _both(x, dy, _tensor((129,), "fp32", 12, 0.2, 1.0)[1:], _tensor((128,), "fp32", 13, 0.2), "bf16")
    assert torch.equal(rt.layer_norm(x), rt.layer_norm(x.contiguous()))


def test_without_weight_or_bias(gpu):
    x, dy = _tensor((3, 50, 96), "bf16", 14, 1.5, 0.3), _tensor((3, 50, 96), "bf16", 15)
    fwd = rt.layer_norm(x, stats=True)
    _check_forward(x, None, None, 1e-5, fwd, "bf16")
    _check_backward(dy, x, fwd[1], fwd[2], None, rt.layer_norm_backward(dy, x, fwd[1], fwd[2]), "bf16")
    w = _tensor((96,), "fp32", 16, 0.2, 1.0)
    fwd = rt.layer_norm(x, w, stats=True)
    _check_forward(x, w, None, 1e-5, fwd, "bf16")
    _check_backward(dy, x, fwd[1], fwd[2], w, rt.layer_norm_backward(dy, x, fwd[1], fwd[2], w, bias=False), "bf16", False)


def test_equal_and_shifted_rows(gpu):
    """Rows of one value have no variance (y = bias, rstd = eps^-1/2); a large mean does not swallow it."""
    import torch

    x = torch.full((6, 320), 3.0, device="cuda")
    x[3:] = 4096.0 + torch.arange(320, device="cuda") / 64
    w, b = _tensor((320,), "fp32", 17, 0.2, 1.0), _tensor((320,), "fp32", 18)
    y, mean, rstd = rt.layer_norm(x, w, b, eps=1e-6, stats=True)
    assert torch.equal(y[:3], b.expand(3, 320)) and (mean[:3] == 3.0).all()
    assert (rstd[:3] - 1000.0).abs().max() <= 1000.0 * 4 * U
    _check_forward(x, w, b, 1e-6, (y, mean, rstd), "fp32")


def test_no_rows_give_zero_sums(gpu):
    import torch

    w = torch.ones(2, 64, device="cuda")
    x = torch.empty((2, 0, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.empty((2, 0), device="cuda")
    assert rt.layer_norm(x, w).shape == x.shape
    for weight in (w, w[0]):
        dx, dw, db = rt.layer_norm_backward(x, x, s, s, weight)
        assert dx.shape == x.shape and dw.shape == weight.shape and (dw == 0).all() and (db == 0).all()


def test_a_row_that_is_not_finite_stays_in_its_row(gpu):
    import torch

    for W in (64, 65, 1152, 4096):
        x, dy = _tensor((70, W), "fp32", 19), _tensor((70, W), "fp32", 20)
        y, mean, rstd = rt.layer_norm(x, stats=True)
        dx = rt.layer_norm_backward(dy, x, mean, rstd)[0]
        x[33, W - 1] = float("nan")
        yb, mb, rb = rt.layer_norm(x, stats=True)
        dxb = rt.layer_norm_backward(dy, x, mb, rb)[0]
        rest = torch.arange(70, device="cuda") != 33
        assert torch.isnan(yb[33]).all() and torch.isnan(dxb[33]).all()
        assert torch.equal(yb[rest], y[rest]) and torch.equal(dxb[rest], dx[rest])


def test_equal_calls_give_equal_bits(gpu):
    import torch

    x, dy = _tensor((9000, 64), "bf16", 21), _tensor((9000, 64), "bf16", 22)
    w = _tensor((64,), "fp32", 23)
    y, mean, rstd = rt.layer_norm(x, w, stats=True)
    first = rt.layer_norm_backward(dy, x, mean, rstd, w)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, rt.layer_norm_backward(dy, x, mean, rstd, w)))


def test_gradient_of_the_library_forward_is_a_difference(gpu):
    """Differences of the library's own fp32 forward along one direction, against its gradient."""
    import torch

    x, dy, v = (_tensor((4, 96), "fp32", s) for s in (24, 25, 26))
    w = _tensor((96,), "fp32", 27, 0.2, 1.0)
    _, mean, rstd = rt.layer_norm(x, w, stats=True)
    dx = rt.layer_norm_backward(dy, x, mean, rstd, w)[0]
    h = 2.0 ** -6
    up, down = (rt.layer_norm(x + s * h * v, w).double() for s in (1, -1))
    num = float(((up - down) * dy.double()).sum() / (2 * h))
    # third derivatives of a row of unit scale: h^2 / 6 times their size (below 10) for 384 elements' sum, and
    # 2^-22 / h of rounding for each
    assert abs(num - float((dx.double() * v.double()).sum())) <= 384 * (10 * h * h / 6 + U * 4 / h)


def test_workspace_too_small_is_refused(gpu):
    from paper_2505_22918_amd import _lib

    dims = _lib.RtNormDims(1, 1, 64, 64, _lib.RT_BF16, _lib.RT_F32, 1)
    need = ctypes.c_int64()
    assert gpu.rt_layer_norm_backward_workspace(dims, ctypes.byref(need)) == _lib.RT_OK and need.value > 0
