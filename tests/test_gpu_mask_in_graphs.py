"""Masks and their transposes in captured graphs: the gradients of a replay belong to one mask, the one that the arrays
hold then, whatever eager calls did in between."""

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


def _arrays(n, keep, seed):
    import torch

    return tuple(torch.tensor(x, dtype=torch.int32).cuda() for x in _csr(n, keep, seed))


def _grads(q, k, v, d_o, mask, **kw):
    return rt.attn_sparse_backward(q, k, v, *rt.attn_sparse(q, k, v, mask), d_o, mask, **kw)


def _fresh(q, k, v, d_o, n, keep, seed):
    return _grads(q, k, v, d_o, rt.BlockMask.from_csr(*_csr(n, keep, seed), 64))


def _equal(got, want):
    import torch

    torch.cuda.synchronize()
    return all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n", [16, 700])
def test_a_captured_gradient_follows_the_mask(gpu, n):
    """An eager call, a capture, then the mask is rewritten and another eager call made; what it drops is given out
    again.  Each replay is of the mask as it is then."""
    import torch

    q, k, v, d_o = (_bf16(1, 1, n * 64, 64, seed=s) for s in range(4))
    mask = rt.BlockMask.from_csr(*_csr(n, 4, 0), 64)
    assert _equal(_grads(q, k, v, d_o, mask), _fresh(q, k, v, d_o, n, 4, 0))
    outs = [torch.empty_like(q) for _ in range(3)]
    size = mask.transposed().col_idx.numel()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _grads(q, k, v, d_o, mask, out=outs)
    others = []
    for seed in (0, 1, 2):
        want = _fresh(q, k, v, d_o, n, 4, seed)
        mask.col_idx.copy_(torch.tensor(_csr(n, 4, seed)[1], dtype=torch.int32))
        assert _equal(_grads(q, k, v, d_o, mask), want)
        others += [torch.full((size,), -1, dtype=torch.int32, device="cuda") for _ in range(4)]
        for t in outs:
            t.zero_()
        g.replay()
        assert _equal(outs, want), seed
        assert _equal(_grads(q, k, v, d_o, mask), want), seed
    assert all(bool((x == -1).all()) for x in others)
