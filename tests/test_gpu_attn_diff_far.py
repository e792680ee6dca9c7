"""Differential attention of scores far from zero, to the ends of fp32's range: products of powers of two, exact in fp32, whose
softmax is known: keys that share the largest score share the weight, the others have none."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import heads as oh
from test_gpu_attn_diff import _lens, _np, _within

pytestmark = pytest.mark.gpu

# (single tokens and up to 16 queries, whole and in parts; shared keys, whole and in parts; tiles of 128 queries, whole and in parts)
SIZES = [(1, 1, 40), (1, 16, 300), (1, 9, 3000), (1, 17, 300), (1, 200, 300), (1, 33, 1000), (1, 1, 5), (60, 200, 300), (1, 124, 1405)]


@pytest.mark.parametrize("exponent", [12, 17, 24, 40, 80, 100, 120])
@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("H,Tq,Tk", SIZES)
def test_far_scores(gpu, H, Tq, Tk, D, exponent):
    import torch

    print(f"[diff far] H={H} Tq={Tq} Tk={Tk} D={D} 2^{exponent}", flush=True)
    g = torch.Generator().manual_seed(exponent)
    v = torch.randn((2, H, Tk, 2 * D), generator=g).bfloat16()
    lam = torch.full((H,), 0.5)
    # scores of +- 2^exponent and twice that for even rows, 0 for odd ones; negative in the second sample and the second map
    q, k = torch.zeros((2, 2 * H, Tq, D)), torch.ones((2, 2 * H, Tk, 1)) * 2.0 ** (exponent // 2)
    q[:, :, ::2, 0] = 2.0 ** (exponent - exponent // 2)
    tops = [sorted({Tk // 3, Tk - 2}), [Tk // 2]]  # of each map
    for m in range(2):
        for b in range(2):
            two = torch.zeros(Tk, dtype=torch.bool)
            two[tops[m]] = True
            sign = -1.0 if (b or m) else 1.0
            k[b, m::2, :, 0] *= sign * torch.where(two == (sign > 0), 2.0, 1.0)
    k = torch.cat([k, torch.zeros((2, 2 * H, Tk, D - 1))], -1)
    q, k, v, lam = q.bfloat16().cuda(), k.bfloat16().cuda(), v.cuda(), lam.cuda()
    lens = [Tk, Tk - 1]
    for used in (None, _lens(lens)):
        out = rt.attn_diff(q, k, v, lam, k_lens=used)
        assert torch.equal(rt.attn_diff(q, k, v, lam, k_lens=used, stats=False), out[0])
        o, o2, top, total = (_np(x) for x in out)
        for b in range(2):
            n = Tk if used is None else lens[b]
            for h in sorted({0, H - 1}):
                V = _np(v)[b, h]
                P = [V[t].mean(0) for t in tops]
                # results rounded by half a step of bf16, behind sums in fp32 of weights that are exact
                near = 4 * 2.0 ** -24 * np.abs(V).max()
                for x, r in ((o[b, h, ::2], P[0] - 0.5 * P[1]), (o2[b, h, ::2], P[1])):
                    assert np.all(np.abs(x - r) <= 2.0 ** -8 * np.abs(r) + near)
                for m in range(2):
                    sign = -1.0 if (b or m) else 1.0
                    want = sign * 2.0 ** exponent * (2 if sign > 0 else 1) / D ** 0.5
                    assert np.all(np.abs(top[b, 2 * h + m, ::2] - want) <= 2 * 2.0 ** -24 * abs(want))
                    assert np.all(total[b, 2 * h + m, ::2] == len(tops[m]))
                if Tq > 1:
                    maps = slice(2 * h, 2 * h + 2)
                    ref, tol = oh.forward(_np(q)[b, maps, 1::2], _np(k)[b, maps], V, 0.5, n)
                    for x, r, t in zip((o[b, h, 1::2], o2[b, h, 1::2], top[b, maps, 1::2], total[b, maps, 1::2]), ref, tol):
                        _within(x, r, t, "rows of scores of 0")
