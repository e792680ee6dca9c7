"""Layer norm of more rows than one launch has threads for."""

import pytest

import paper_2505_22918_amd as rt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [1, 2])
def test_more_rows_than_a_launch_takes(gpu, W):
    """2^29 + 4096 rows, 16 lanes each: every piece of 4096 equal rows has the piece's own result."""
    import torch

    piece = torch.randn(4096, W, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    w, b = torch.full((W,), 1.5, device="cuda"), torch.arange(1.0, W + 1.0, device="cuda")
    want, mean, rstd = rt.layer_norm(piece, w, b, stats=True)
    n = (1 << 17) + 1
    x = piece.repeat(n, 1)
    y = torch.zeros_like(x)
    assert rt.layer_norm(x, w, b, out=y) is y
    assert bool((y.view(n, -1) == want.view(1, -1)).all())
    dy = torch.ones_like(x)
    dx = torch.zeros_like(x)
    stats = mean.repeat(n), rstd.repeat(n)
    rt.layer_norm_backward(dy, x, *stats, w, out=dx)
    assert bool((dx.view(n, -1) == rt.layer_norm_backward(dy[:4096], piece, mean, rstd, w)[0].view(1, -1)).all())
