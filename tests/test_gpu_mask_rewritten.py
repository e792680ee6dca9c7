"""Masks whose arrays are written after their first gradient call, in ways that torch's counters do not show."""

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
    return list(range(0, n * keep + 1, keep)), sum(rows, [])


def _col(n, keep, seed):
    import torch

    return torch.tensor(_csr(n, keep, seed)[1], dtype=torch.int32).cuda()


def _grads(x, mask, **kw):
    q, k, v, d_o = x
    return rt.attn_sparse_backward(q, k, v, *rt.attn_sparse(q, k, v, mask), d_o, mask, **kw)


def _same(got, x, n, keep, seed):
    import torch

    want = _grads(x, rt.BlockMask.from_csr(*_csr(n, keep, seed), 64))
    torch.cuda.synchronize()
    return all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.fixture
def x(gpu):
    return [_bf16(1, 2, 1024, 64, seed=s) for s in range(4)]


@pytest.mark.parametrize("inside", [True, False])
def test_a_mask_rewritten_in_inference_mode(x, inside):
    """Inference tensors, and ordinary ones that are written in inference mode."""
    import contextlib

    import torch

    with torch.inference_mode() if inside else contextlib.nullcontext():
        mask = rt.BlockMask.from_csr(*_csr(16, 4, 0), 64)
    for seed in (0, 1, 2):
        with torch.inference_mode():
            mask.col_idx.copy_(_col(16, 4, seed))
            assert _same(_grads(x, mask), x, 16, 4, seed)


def _static(n, keep, made):
    """A mask over buffers that a graph fills from another buffer, and the graph: the mask made before or after the
    capture, or by from_csr."""
    import torch

    rp, ci = (torch.tensor(a, dtype=torch.int32).cuda() for a in _csr(n, keep, 0))
    mask = None
    if made == "csr":
        mask = rt.BlockMask.from_csr(*_csr(n, keep, 0), 64)
        rp, ci = mask.row_ptr, mask.col_idx
    elif made == "before":
        mask = rt.BlockMask(rp, ci, 64, n, n * keep)
    source = ci.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ci.copy_(source)
    return mask or rt.BlockMask(rp, ci, 64, n, n * keep), source, g


@pytest.mark.parametrize("early", [True, False])
@pytest.mark.parametrize("made", ["csr", "before", "after"])
def test_a_graph_that_writes_the_arrays_of_a_mask(x, made, early):
    """Eager calls between the replays, with and without one before the capture."""
    mask, source, g = _static(16, 4, made)
    if early:
        assert _same(_grads(x, mask), x, 16, 4, 0)
    for seed in (1, 2, 3):
        source.copy_(_col(16, 4, seed))
        g.replay()
        for _ in range(2):
            assert _same(_grads(x, mask), x, 16, 4, seed), seed


def test_a_mask_made_by_hand_in_a_capture(x):
    """Its arrays are the graph's own, which every replay writes."""
    import torch

    source = _col(16, 4, 0)
    rp = torch.tensor(_csr(16, 4, 0)[0], dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mask = rt.BlockMask(rp, source + 0, 64, 16, 64)
    for seed in (1, 2, 3):
        source.copy_(_col(16, 4, seed))
        g.replay()
        for _ in range(2):
            assert _same(_grads(x, mask), x, 16, 4, seed), seed


def test_uncounted_writes_and_a_transpose_asked_for(x):
    """Writes through .data leave torch's counters as they are."""
    mask = rt.BlockMask.from_csr(*_csr(16, 4, 0), 64)
    assert _same(_grads(x, mask), x, 16, 4, 0)
    for seed in (1, 2):
        mask.col_idx.data.copy_(_col(16, 4, seed))
        t = mask.transposed(anew=True)
        assert _same(_grads(x, mask), x, 16, 4, seed)
        assert _same(_grads(x, mask, transposed=t), x, 16, 4, seed)


def test_captured_calls_over_a_transpose_that_the_caller_holds(x):
    import torch

    q, k, v, d_o = x
    mask = rt.BlockMask.from_csr(*_csr(16, 4, 0), 64)
    t = mask.transposed()
    stats = rt.attn_sparse(q, k, v, mask)
    outs = [torch.empty_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rt.attn_sparse_backward(q, k, v, *stats, d_o, mask, out=outs, transposed=t)
    for _ in range(3):
        for o in outs:
            o.zero_()
        want = rt.attn_sparse_backward(q, k, v, *stats, d_o, mask)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_what_is_no_transpose_of_the_mask_is_refused(x):
    import torch

    mask = rt.BlockMask.from_csr(*_csr(16, 4, 0), 64)
    t = mask.transposed()
    cut = lambda **kw: rt.BlockMask(**{**{f: getattr(t, f) for f in t.__dataclass_fields__}, **kw})  # noqa: E731
    assert _same(_grads(x, mask, transposed=cut()), x, 16, 4, 0)
    bad = [mask, t.col_idx, rt.BlockMask.from_csr(*_csr(16, 3, 0), 64).transposed(), rt.BlockMask.from_csr(*_csr(32, 4, 0), 32).transposed(),
           cut(row_ptr=t.row_ptr[:-1]), cut(col_idx=t.col_idx[:-1]), cut(col_idx=t.col_idx.long()), cut(nnz=t.nnz + 4096),
           cut(n_masks=2), cut(row_ptr=t.row_ptr.cpu()), cut(col_idx=torch.stack([t.col_idx] * 2, 1)[:, 0])]
    for i, b in enumerate(bad):
        with pytest.raises(ValueError):
            _grads(x, mask, transposed=b)
            print("accepted:", i)
