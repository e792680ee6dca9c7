"""Whether long key lists can be split goes by the mask's blocks, not by how many masks there are."""

import ctypes

import numpy as np
import pytest

from paper_2505_22918_amd import _lib


@pytest.mark.parametrize("n", [41, 55, 83, 96, 97])
@pytest.mark.parametrize("masks", [1, 12])
def test_room_for_parts(n, masks):
    entries = masks * n * 6
    size = ctypes.c_int64()
    assert _lib.load().rt_index_transpose_size(ctypes.byref(_lib.RtBsr(None, None, 64, n, entries, masks)), entries,
                                               ctypes.byref(size)) == _lib.RT_OK
    first = -(-entries // 4) * 4
    assert size.value == first + 4 * (masks * n + 2 * (entries // 16))


@pytest.mark.gpu
@pytest.mark.parametrize("D,block,n", [(64, 64, 55), (72, 64, 83), (64, 32, 96)])
def test_masks_of_each_head_with_a_block_that_all_keep(gpu, D, block, n):
    """Split, and right against the oracle."""
    import paper_2505_22918_amd as rt
    from oracle import gradients as og
    from test_gpu_attn_backward import _compare, _inputs, _masks

    H, T = 3, n * block - 9
    rp, ci = _masks(n, H, 3, n, column=n // 2)
    mask = rt.BlockMask.from_csr(rp, ci, block, n_masks=H)
    plan = mask.transposed().col_idx[-(-len(ci) // 4) * 4:].cpu().numpy().reshape(-1, 4)
    records = plan[H * n + (len(plan) - H * n) // 2:]
    assert sorted(x // n for x in records[:, 0] if x >= 0) == list(range(H))
    dev, host = _inputs(1, H, T, D, n)
    stats = rt.attn_sparse(*dev[:3], mask)
    rows = np.asarray(rp).reshape(H, n + 1)
    _compare(host, stats, rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask),
             lambda b, h: og.token_mask(rows[h], ci, block, T))
