"""One byte less than the layer norm's gradients ask for is refused, on the host."""

import ctypes

import pytest

from paper_2505_22918_amd import _lib

AT = [0x7F0000000000 + i * (1 << 32) for i in range(9)]  # never dereferenced


@pytest.mark.parametrize("n0,n1,W,sets", [(1, 64, 64, 1), (4, 900, 1152, 4), (2, 30, 16384, 1), (3, 5, 129, 3)])
def test_a_byte_too_small(n0, n1, W, sets):
    lib = _lib.load()
    dims = _lib.RtNormDims(n0, n1, 1, W, _lib.RT_BF16, _lib.RT_F32, sets)
    need = ctypes.c_int64()
    assert lib.rt_layer_norm_backward_workspace(dims, ctypes.byref(need)) == _lib.RT_OK and need.value > 0
    s = _lib.Strides(n1 * W, W, W)
    assert lib.rt_layer_norm_backward(AT[0], s, AT[1], s, AT[2], AT[3], AT[4], dims, AT[5], s, AT[6], AT[7], AT[8],
                                      need.value - 1, None) == _lib.RT_ECAPACITY
    assert f"{need.value} needed" in lib.rt_last_error().decode()
