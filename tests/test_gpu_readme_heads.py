"""The calls of rotary positions and differential attention as the README writes them: run as they stand, a batch of two, against
the same layers in 64 bits by autograd."""

import os

import pytest

import paper_2505_22918_amd as rt

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _block(first):
    """The code block that begins with this comment."""
    with open(README) as f:
        blocks = f.read().split("```python\n")[1:]
    return next(b.split("```")[0] for b in blocks if b.startswith(first))


def _near(got, ref, roundings):
    # independent roundings of half a bf16 step at most (2^-8 / sqrt(3) each) on the way to a result, four times their norm
    err = float((got.double().cpu() - ref).norm() / ref.norm())
    assert err <= 4 * (roundings / 3) ** 0.5 * 2.0 ** -8, err


def test_packed_projection_to_attention_and_back(gpu):
    import torch

    B, T, H, D = 2, 70, 3, 64
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((B, T, 3, H, D), generator=g).bfloat16().cuda()
    d_o = torch.randn((B, H, T, D), generator=g).bfloat16().cuda()
    positions = torch.stack([torch.arange(T) // 20, torch.arange(T) % 20 // 5, torch.arange(T) % 5], -1).cuda()
    names = dict(rt=rt, torch=torch, qkv=qkv, positions=positions, d_o=d_o)
    exec(_block("# queries and keys out of a packed projection"), names)

    leaf = qkv.double().cpu().requires_grad_()
    plan = names["plan"]
    angle = positions.cpu().double()[:, plan.axis.cpu().long()] * plan.freq.cpu()
    turn = torch.polar(torch.ones_like(angle), angle)
    x = leaf.permute(2, 0, 3, 1, 4)
    q, k = (torch.view_as_real(torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2) for y in x[:2])
    o = (q @ k.transpose(2, 3) / D ** 0.5).softmax(-1) @ x[2]
    (o * d_o.double().cpu()).sum().backward()
    _near(names["o"], o.detach(), 4)  # queries, keys, probabilities, the result
    for i in range(3):
        _near(names["d_qkv"][:, :, i], leaf.grad[:, :, i], 8)  # these, dS, the gradient, turned back


def test_differential_attention_and_its_cache(gpu):
    import torch

    B, H, T, D = 2, 3, 70, 64
    g = torch.Generator().manual_seed(4)
    n = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    q, k, v, d_o = n(B, 2 * H, T, D), n(B, 2 * H, T, D), n(B, H, T, 2 * D), n(B, H, T, 2 * D)
    lam, lens = (0.5 + 0.1 * torch.randn(H, generator=g)).cuda(), torch.tensor([T, 41], dtype=torch.int32, device="cuda")
    names = dict(rt=rt, torch=torch, q=q, k=k, v=v, lam=lam, lens=lens, d_o=d_o, q1=q[:, :, :1].contiguous(), cache_k=k, cache_v=v)
    exec(_block("# two softmax maps to a head"), names)

    leaves = [t.double().cpu().requires_grad_() for t in (q, k, v, lam)]
    Q, K, V, L = leaves
    S = (Q @ K.transpose(2, 3) / D ** 0.5).masked_fill(torch.arange(T) >= lens.cpu()[:, None, None, None], -float("inf"))
    A = S.softmax(-1).unflatten(1, (H, 2))
    o = (A[:, :, 0] - L[:, None, None] * A[:, :, 1]) @ V
    (o * d_o.double().cpu()).sum().backward()
    _near(names["o"], o.detach()[:, :, :1], 4)
    for got, leaf in zip((names["dq"], names["dk"], names["dv"], names["d_lam"]), leaves):
        _near(got, leaf.grad, 8)
