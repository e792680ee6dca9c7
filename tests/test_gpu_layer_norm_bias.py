"""Layer norm with a bias and no weight, forward and gradients, against the 64-bit oracle; its bounds are those of
test_gpu_layer_norm.py."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from test_gpu_layer_norm import COL_DEPTH, U, _check_forward, _np, _tensor
from oracle import gradients as og

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,own", [("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("W", [64, 129, 1152])
@pytest.mark.parametrize("sets", [False, True])
def test_bias_alone(gpu, sets, W, dtype, own):
    B, N = 3, 41
    x, dy = _tensor((B, N, W), dtype, 1, 1.5, 0.3), _tensor((B, N, W), dtype, 2)
    b = _tensor((B, W) if sets else (W,), own, 3)
    out = rt.layer_norm(x, None, b, stats=True)
    _check_forward(x, None, b, 1e-5, out, dtype)
    dx, dw, db = rt.layer_norm_backward(dy, x, *out[1:], bias=b)
    assert dw is None and db.shape == b.shape and db.dtype.itemsize == 4
    dY = _np(dy).reshape(B, N, W)
    over = 1 if sets else (0, 1)
    assert (np.abs(_np(db) - dY.sum(over)) <= COL_DEPTH * U * np.abs(dY).sum(over)).all()
    assert (dx == rt.layer_norm_backward(dy, x, *out[1:])[0]).all()


def test_bias_of_the_forward_call_beside_a_weight(gpu):
    x, dy, w, b = _tensor((5, 7, 72), "bf16", 1), _tensor((5, 7, 72), "bf16", 2), _tensor((72,), "fp32", 3), _tensor((72,), "fp32", 4)
    _, mean, rstd = rt.layer_norm(x, w, b, stats=True)
    want = rt.layer_norm_backward(dy, x, mean, rstd, w)
    got = rt.layer_norm_backward(dy, x, mean, rstd, w, bias=b)
    assert all((a == c).all() for a, c in zip(got, want))
    for no in (False, None, 0):
        assert rt.layer_norm_backward(dy, x, mean, rstd, w, bias=no)[2] is None
    assert (rt.layer_norm_backward(dy, x, mean, rstd, w, bias=1)[2] == want[2]).all()
    assert rt.layer_norm_backward(dy, x, mean, rstd)[1:] == (None, None)
    for bad in (b[:71], b.half(), b.cpu(), _tensor((5, 72), "fp32", 5)):
        with pytest.raises(ValueError):
            rt.layer_norm_backward(dy, x, mean, rstd, w, bias=bad)
