"""Sizes that one launch of the training calls cannot take (2^32 threads) are refused on the host."""

import ctypes

import pytest

from paper_2505_22918_amd import _lib

AT = [0x7F0000000000 + i * (1 << 38) for i in range(20)]  # never dereferenced
ROOM = 1 << 36


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _bsr(i, block, n, nnz, masks):
    return _lib.RtBsr(AT[i], AT[i + 1], block, n, nnz, masks)


@pytest.mark.parametrize("B,H,T", [(1 << 10, 1 << 13, 1), (1 << 8, (1 << 15) - 1, 65), (64, 8192, 1024), (8, 8, 1 << 23)])
def test_rows_past_a_launch(lib, B, H, T):
    dims = _lib.RtDims(B, H, T, 64)
    assert lib.rt_attn_full_backward(*AT[:7], dims, *AT[7:11], ROOM, None) == _lib.RT_EINVAL
    assert "too many rows" in lib.rt_last_error().decode()
    n = -(-T // 64)
    mask, t = _bsr(11, 64, n, n, 1), _bsr(13, 64, n, n, 1)
    got = lib.rt_attn_sparse_backward(*AT[:7], dims, ctypes.byref(mask), ctypes.byref(t), None, 0.0, *AT[7:10], None, AT[10],
                                      ROOM, None)
    assert got == _lib.RT_EINVAL and "too many" in lib.rt_last_error().decode()


def test_mask_rows_past_a_launch(lib):
    n, masks = 64, 1 << 20
    mask, t = _bsr(0, 64, n, n * masks, masks), _bsr(2, 64, n, n * masks, masks)
    size = ctypes.c_int64()
    assert lib.rt_index_transpose_size(ctypes.byref(mask), n * masks, ctypes.byref(size)) == _lib.RT_EINVAL
    assert "too many mask rows" in lib.rt_last_error().decode()
    assert lib.rt_index_transpose(ctypes.byref(mask), 64 * n, ctypes.byref(t), None) == _lib.RT_EINVAL
    assert "too many mask rows" in lib.rt_last_error().decode()
