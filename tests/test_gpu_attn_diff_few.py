"""Differential attention of up to 16 queries takes probabilities in two bf16 pieces: a bound on its outputs that one piece does
not meet."""

import numpy as np
import pytest

import diff_plans
import paper_2505_22918_amd as rt
from oracle import heads as oh
from test_gpu_attn_diff import _inputs, _lens, _np, _within

# whole and in parts, with keys that end inside a tile; scores spread by SHARP, so that a few keys of thousands have most of the
# weight: the bound allows fp32 sums a rounding a key, beside which what one piece loses shows there alone
SHARP = 3.0
SIZES = [(1, 2, 16, 300, None), (1, 1, 1, 500, None), (2, 1, 5, 700, (700, 331)), (1, 1, 9, 3000, None), (3, 2, 15, 2100, (2100, 40, 1777))]


def _bf16(x):
    """float32 rounded to the nearest bf16, ties to even."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return diff_plans.build(str(tmp_path_factory.mktemp("diff_few")))


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("B,H,Tq,Tk,lens", SIZES)
def test_one_piece_does_not_meet_the_bound(lib, B, H, Tq, Tk, lens, D):
    """On the CPU, in 64 bits but for the rounding of probabilities and of the result."""
    import torch

    assert diff_plans.forward(lib, B, H, Tq, Tk, D, lens is not None)[0] == "few"
    g = torch.Generator().manual_seed(Tk)
    q, k, v = ((torch.randn(s, generator=g) * f).bfloat16().double().numpy() for s, f in (((2, Tq, D), SHARP), ((2, Tk, D), 1), ((Tk, 2 * D), 1)))
    (o, o2, m, l), (tol, *_) = oh.forward(q, k, v, 0.5, Tk, pieces=2, waves=4)
    for pieces in (1, 2):
        out = []
        for i in range(2):
            p = np.exp(q[i] @ k[i].T / np.sqrt(D) - m[i][:, None])
            hi = _bf16(p)
            out.append((hi + (_bf16(p - hi) if pieces == 2 else 0.0)) @ v / l[i][:, None])
        err = np.abs(_bf16(out[0] - 0.5 * out[1]) - o)
        assert np.all(err <= tol) == (pieces == 2)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("B,H,Tq,Tk,lens", SIZES)
def test_few_queries(gpu, B, H, Tq, Tk, lens, D):
    print(f"[diff few] B={B} H={H} Tq={Tq} Tk={Tk} D={D} lens={lens}", flush=True)
    q, k, v, _, lam = _inputs(B, H, Tq, Tk, D, Tk, SHARP)
    o, o2, m, l = (_np(x) for x in rt.attn_diff(q, k, v, lam, k_lens=_lens(lens)))
    q, k, v, lam = (_np(x) for x in (q, k, v, lam))
    for b in range(B):
        for h in range(H):
            maps = slice(2 * h, 2 * h + 2)
            ref, tol = oh.forward(q[b, maps], k[b, maps], v[b, h], lam[h], Tk if lens is None else lens[b], pieces=2, waves=4)
            for x, r, t, name in zip((o[b, h], o2[b, h], m[b, maps], l[b, maps]), ref, tol, ("o", "o2", "m", "l")):
                _within(x, r, t, (name, b, h))
