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
