"""The transpose that a BlockMask keeps: never one of other contents, never memory given out again under a call."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt

pytestmark = pytest.mark.gpu


def _bf16(*shape, seed=0):
    import torch

    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def _csr(n, keep, seed):
    rng = np.random.default_rng(seed)
    rows = [sorted(rng.choice(n, size=keep, replace=False).tolist()) for _ in range(n)]
    return np.arange(0, n * keep + 1, keep), sum(rows, [])


def _grads(q, k, v, d_o, mask):
    return rt.attn_sparse_backward(q, k, v, *rt.attn_sparse(q, k, v, mask), d_o, mask)


def test_a_mask_that_a_graph_makes_is_transposed_each_time(gpu):
    """dynamic_index captured alone: each replay writes another mask into the same arrays."""
    import torch

    T = 700
    q, k, v, d_o = (_bf16(1, 2, T, 64, seed=s) for s in range(4))
    rt.dynamic_index(q, k, 64, 4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mask = rt.dynamic_index(q, k, 64, 4)
    for i in range(3):
        q.copy_(_bf16(1, 2, T, 64, seed=10 + i))
        g.replay()
        for _ in range(2):
            got = _grads(q, k, v, d_o, mask)
            want = _grads(q, k, v, d_o, rt.dynamic_index(q, k, 64, 4))
            assert all(torch.equal(a, b) for a, b in zip(got, want)), f"replay {i}"


def test_a_rewritten_mask_is_transposed_anew(gpu):
    import torch

    q, k, v, d_o = (_bf16(1, 2, 1024, 64, seed=s) for s in range(4))
    mask = rt.BlockMask.from_csr(*_csr(16, 4, 0), 64)
    _grads(q, k, v, d_o, mask)
    torch.cuda.synchronize()
    assert mask.transposed() is mask.transposed()
    for seed in (1, 2):
        rp, ci = _csr(16, 4, seed)
        mask.col_idx.copy_(torch.tensor(ci, dtype=torch.int32))
        got, want = _grads(q, k, v, d_o, mask), _grads(q, k, v, d_o, rt.BlockMask.from_csr(rp, ci, 64))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_memory_of_a_mask_dropped_under_another_stream(gpu):
    """Built on one stream, used on a second whose work is still under way when the mask goes: the transpose's memory
    stays taken until that work has ended."""
    import torch

    q, k, v, d_o = (_bf16(1, 2, 1024, 64, seed=s) for s in range(4))
    rp, ci = _csr(16, 4, 0)
    mask = rt.BlockMask.from_csr(rp, ci, 64)
    stats = rt.attn_sparse(q, k, v, mask)
    want = rt.attn_sparse_backward(q, k, v, *stats, d_o, mask)
    t = mask.transposed()
    size, at = t.col_idx.numel(), t.col_idx.data_ptr()
    held = mask.row_ptr, mask.col_idx  # the caller's own arrays are the caller's to keep
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # about 0.1 s
        got = rt.attn_sparse_backward(q, k, v, *stats, d_o, mask)
        busy = side.record_event()
    del t, mask
    others = [torch.full((size,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
    assert not busy.query(), "the side stream ended before the check"
    assert all(not o.data_ptr() <= at < o.data_ptr() + 4 * size for o in others)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(held) == 2


def test_masks_under_inference_mode(gpu):
    import torch

    q, k, v, d_o = (_bf16(1, 2, 1024, 64, seed=s) for s in range(4))
    csr = _csr(16, 4, 3)
    want = _grads(q, k, v, d_o, rt.BlockMask.from_csr(*csr, 64))
    with torch.inference_mode():
        mask = rt.BlockMask.from_csr(*csr, 64)
        for _ in range(2):
            assert all(torch.equal(a, b) for a, b in zip(_grads(q, k, v, d_o, mask), want))
