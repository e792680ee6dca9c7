"""Values of one map that are not finite stay out of the other map's statistics, output and gradients."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import heads as oh
from test_gpu_attn_diff import _inputs, _np, _within

pytestmark = pytest.mark.gpu

# (single tokens and up to 16 queries, whole and in parts; shared keys; tiles of 128 queries)
SIZES = [(1, 1, 40), (1, 9, 3000), (2, 16, 300), (2, 17, 300), (1, 100, 70), (2, 200, 300), (1, 300, 40), (1, 129, 700), (2, 1040, 1040), (40, 300, 130)]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("H,Tq,Tk", SIZES)
def test_a_bad_key_stays_in_its_map(gpu, H, Tq, Tk, D, bad):
    print(f"[diff other map] H={H} Tq={Tq} Tk={Tk} D={D} bad={bad}", flush=True)
    q, k, v, _, lam = _inputs(1, H, Tq, Tk, D, Tq + Tk)
    h = H - 1  # a key of the last head
    maps = slice(2 * h, 2 * h + 2)
    ref, tol = oh.forward(_np(q)[0, maps], _np(k)[0, maps], _np(v)[0, h], _np(lam)[h], Tk)
    for m in (0, 1):
        kb = k.clone()
        kb[0, 2 * h + m, Tk // 3, D - 3] = bad
        o, o2, top, total = (_np(x) for x in rt.attn_diff(q, kb, v, lam))
        _within(top[0, 2 * h + 1 - m], ref[2][1 - m], tol[2][1 - m], "max")
        _within(total[0, 2 * h + 1 - m], ref[3][1 - m], tol[3][1 - m], "sum")
        if m == 0:
            _within(o2[0, h], ref[1], tol[1], "o2")
        if np.isnan(bad):  # (an infinite key may also give scores of -inf, whose weight is 0)
            assert np.isnan(o[0, h]).all() and np.isnan(total[0, 2 * h + m]).all()


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("Tq,Tk", [(9, 300), (16, 3000), (100, 70), (200, 300), (1040, 1040)])
def test_a_bad_query_stays_in_its_map(gpu, Tq, Tk, D):
    q, k, v, _, lam = _inputs(1, 1, Tq, Tk, D, Tq + Tk + 1)
    ref, tol = oh.forward(_np(q)[0], _np(k)[0], _np(v)[0, 0], _np(lam)[0], Tk)
    q[0, 0, Tq // 2, 7] = float("nan")
    _, o2, top, total = (_np(x)[0] for x in rt.attn_diff(q, k, v, lam))
    _within(o2[0], ref[1], tol[1], "o2")
    _within(top[1], ref[2][1], tol[2][1], "max")
    _within(total[1], ref[3][1], tol[3][1], "sum")


# ---- gradients: those of the second map's queries and keys do not depend on the first (dS_2 = -lam P_2 (dA - dO . O_2)) ----

# (in one launch, by four waves and eight, whole and in parts)
GRAD_SIZES = [(1, 1, 40), (1, 9, 3000), (2, 17, 300), (1, 100, 70), (2, 200, 300), (1, 300, 40), (1, 129, 700), (2, 1040, 1040), (40, 300, 130)]


def _second_map(q, k, v, do, lam, bad_q, bad_k):
    """dq and dk of the last head's second map and its dlam with values of the first that are not finite, against those
    without."""
    n = [_np(x) for x in (q, k, v, do, lam)]
    H, Tk, h = v.shape[1], v.shape[2], v.shape[1] - 1
    maps = slice(2 * h, 2 * h + 2)
    o = _np(rt.attn_diff(q, k, v, lam)[0])[0, h]
    out = rt.attn_diff(bad_q, bad_k, v, lam)
    dq, dk, _, dlam = (_np(x) for x in rt.attn_diff_backward(bad_q, bad_k, v, *out, do, lam))
    (_, _, m, l), _ = oh.forward(n[0][0, maps], n[1][0, maps], n[2][0, h], n[4][h], Tk)
    m[1], l[1] = (_np(x)[0, 2 * h + 1] for x in out[2:])
    o2 = _np(out[1])[0, h]
    assert np.isfinite(o2).all() and np.isfinite(l).all()
    ref, tol = oh.backward(n[0][0, maps], n[1][0, maps], n[2][0, h], o, o2, m, l, n[3][0, h], n[4][h], Tk)
    _within(dq[0, 2 * h + 1], ref[0][1], tol[0][1], "dq")
    _within(dk[0, 2 * h + 1], ref[1][1], tol[1][1], "dk")
    _within(dlam[h], ref[3], tol[3], "dlam")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("H,Tq,Tk", GRAD_SIZES)
def test_gradients_of_the_second_map_without_the_first(gpu, H, Tq, Tk, D, bad):
    print(f"[diff other map] gradients H={H} Tq={Tq} Tk={Tk} D={D} bad={bad}", flush=True)
    q, k, v, do, lam = _inputs(1, H, Tq, Tk, D, Tq + Tk)
    bad_k, bad_q = k.clone(), q.clone()
    bad_k[0, 2 * H - 2, Tk // 3, D - 3] = bad
    bad_q[0, 2 * H - 2, Tq // 2, 7] = bad
    _second_map(q, k, v, do, lam, q, bad_k)
    _second_map(q, k, v, do, lam, bad_q, k)
