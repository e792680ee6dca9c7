"""Differential attention and its gradients by each kernel and plan that a call can take, over walks of several stages,
against the fp64 oracle.  test_diff_plans.py checks on the CPU that these sizes take the plans that they are here for."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import heads as oh
from test_gpu_attn_diff import _inputs, _lens, _np, _within

pytestmark = pytest.mark.gpu

# B, H, Tq, Tk, D, numbers of keys or None; the forward kernel (tile: 128 queries to four waves, keys: the waves share 32
# queries' keys) and whether it takes the keys in parts; waves to a tile of the gradients, and the walks in parts
CASES = [
    (1, 35, 700, 700, 64, None, "tile", False, 4, ""),
    (1, 35, 700, 700, 72, None, "tile", False, 4, ""),
    (3, 20, 200, 300, 64, (300, 7, 129), "tile", False, 4, ""),
    (3, 20, 200, 300, 72, (40, 300, 129), "tile", False, 4, ""),
    (1, 1, 124, 1405, 64, None, "tile", True, 8, "q"),
    (2, 1, 50, 1407, 64, (300, 1407), "tile", True, 4, "q"),
    (1, 2, 38, 1140, 72, (1005,), "tile", True, 4, "q"),
    (2, 4, 1055, 3733, 64, None, "tile", True, 4, "q"),
    (3, 3, 897, 2568, 72, None, "tile", True, 4, "q"),
    (8, 2, 823, 2975, 64, (700, 2975, 0, 1, 2001, 2975, 64, 1299), "tile", True, 8, "q"),
    (2, 2, 2747, 2747, 72, (2747, 1100), "tile", True, 4, "kq"),
    (1, 2, 1008, 1008, 64, None, "keys", False, 8, "kq"),
    (1, 2, 1071, 1071, 72, None, "keys", False, 8, "kq"),
    (1, 4, 1108, 346, 64, None, "keys", False, 8, "k"),
    (4, 1, 972, 264, 72, None, "keys", False, 8, "k"),
    (1, 4, 217, 1003, 64, None, "keys", False, 8, "q"),
    (2, 1, 241, 2056, 72, None, "keys", True, 8, "q"),
    (2, 2, 1002, 1002, 64, (610, 1002), "keys", False, 8, "kq"),
    (3, 1, 1070, 1070, 72, (1070, 0, 333), "keys", False, 8, "kq"),
    (4, 2, 928, 356, 64, (356, 100, 1, 0), "keys", False, 8, "k"),
    (3, 2, 1029, 290, 72, (131, 290, 128), "keys", False, 8, "k"),
    (4, 1, 288, 2576, 64, (2576, 1000, 64, 65), "keys", True, 8, "q"),
    (3, 2, 205, 919, 72, (919, 500, 129), "keys", False, 8, "q"),
    (2, 2, 729, 729, 64, (729, 390), "keys", False, 4, "kq"),
    (2, 2, 730, 730, 72, (400, 730), "keys", False, 4, "kq"),
    (2, 4, 560, 240, 64, (240, 100), "keys", False, 4, "k"),
    (4, 1, 1167, 209, 72, (0, 209, 64, 150), "keys", False, 4, "k"),
    (4, 1, 190, 1285, 72, (1285, 1, 640, 700), "keys", True, 4, "q"),
]


def _heads(B, H, Tq, Tk):
    """Which (sample, head) pairs are looked at: all of a small call's, the corners and one between of a large one's."""
    if B * H * Tq * Tk <= 1 << 22:
        return [(b, h) for b in range(B) for h in range(H)]
    return sorted({(0, 0), (B // 2, H // 2), (B - 1, H - 1)})


def _check(B, H, Tq, Tk, D, lens, q, k, v, do, lam):
    import torch

    used = None if lens is None else list(lens)
    lens = _lens(used)
    out = rt.attn_diff(q, k, v, lam, k_lens=lens)
    assert torch.equal(rt.attn_diff(q, k, v, lam, k_lens=lens, stats=False), out[0])
    got = rt.attn_diff_backward(q, k, v, *out, do, lam, k_lens=lens)
    n = [_np(x) for x in (q, k, v, do, lam)]
    o, o2, m, l = (_np(x) for x in out)
    dq, dk, dv, dlam = (_np(x) for x in got)
    for b, h in _heads(B, H, Tq, Tk):
        two, keys = slice(2 * h, 2 * h + 2), Tk if used is None else used[b]
        ref, tol = oh.forward(n[0][b, two], n[1][b, two], n[2][b, h], n[4][h], keys)
        for x, r, t, name in zip((o[b, h], o2[b, h], m[b, two], l[b, two]), ref, tol, ("o", "o2", "m", "l")):
            _within(x, r, t, (name, b, h))
        ref, tol = oh.backward(n[0][b, two], n[1][b, two], n[2][b, h], o[b, h], o2[b, h], m[b, two], l[b, two], n[3][b, h], n[4][h], keys)
        for x, r, t, name in zip((dq[b, two], dk[b, two], dv[b, h]), ref, tol, ("dq", "dk", "dv")):
            _within(x, r, t, (name, b, h))
    # dlam: of all samples, from the second outputs that the gradients were given (products and sums of 2 D values in fp32)
    terms = (n[3] * o2).sum(-1)
    size = np.abs(n[3] * o2).sum((0, 2, 3))
    assert np.all(np.abs(dlam + terms.sum((0, 2))) <= ((2 * D + 8) * size + np.abs(dlam)) * 2.0 ** -24 + 1e-30)
    if used is not None:
        for b, keys in enumerate(used):
            assert not got[1][b, :, keys:].any() and not got[2][b, :, keys:].any()
    return out, got


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:5]) + ("-lens" if c[5] else ""))
def test_plans(gpu, case):
    import torch

    B, H, Tq, Tk, D, lens = case[:6]
    print(f"[diff plans] B={B} H={H} Tq={Tq} Tk={Tk} D={D} lens={lens}", flush=True)
    q, k, v, do, lam = _inputs(B, H, Tq, Tk, D, Tq + Tk)
    out, got = _check(B, H, Tq, Tk, D, lens, q, k, v, do, lam)
    if lens is not None:  # what lies past a sample's keys is not used
        for b, n in enumerate(lens):
            k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
        on = _lens(lens)
        assert all(torch.equal(x, y) for x, y in zip(out, rt.attn_diff(q, k, v, lam, k_lens=on)))
        assert all(torch.equal(x, y) for x, y in zip(got, rt.attn_diff_backward(q, k, v, *out, do, lam, k_lens=on)))


# scores that rise by hundreds from tile to tile, fall again, and lie far below zero: the running max moves in the middle of
# a walk, in tiles of 128 queries whole and in parts , and in gradients of four waves and of eight
RAMPS = [(1, 60, 200, 400, 64, "tile", False, 4, ""), (1, 60, 200, 400, 72, "tile", False, 4, ""), (1, 1, 124, 1405, 64, "tile", True, 8, "q"),
         (3, 3, 897, 2568, 72, "tile", True, 4, "q"), (1, 2, 1008, 1008, 64, "keys", False, 8, "kq"), (1, 2, 1071, 1071, 72, "keys", False, 8, "kq")]


@pytest.mark.parametrize("B,H,Tq,Tk,D", [c[:5] for c in RAMPS])
def test_running_max_moves_in_every_kernel(gpu, B, H, Tq, Tk, D):
    import torch

    print(f"[diff plans] ramp B={B} H={H} Tq={Tq} Tk={Tk} D={D}", flush=True)
    q, k, v, do, lam = _inputs(B, H, Tq, Tk, D, 9)
    ramp = torch.linspace(-40, 60, Tk, device="cuda")
    ramp[Tk // 2:3 * Tk // 4] = -50
    q[..., 0], k[..., 0] = 4.0, ramp.bfloat16()
    k[:, 1::2, :, 0] = ramp.flip(0).bfloat16()
    _check(B, H, Tq, Tk, D, None, q, k, v, do, lam)
