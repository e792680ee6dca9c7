"""Plans of rotary positions: scaled frequencies, and the grids of the workloads (CPU)."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from paper_2505_22918_amd import schedule, synth


def test_scaled_frequencies():
    import math

    f = [10000.0 ** (-2 * i / 64) for i in range(32)]
    same = lambda a, b: np.allclose(a.freq.numpy(), b, rtol=1e-14, atol=0)  # noqa: E731
    kw = dict(device="cpu")
    assert same(rt.rope_plan(64, **kw), f) and rt.rope_plan(64, **kw).amplitude == 1.0
    assert same(rt.rope_plan(64, scaling="linear", factor=4.0, **kw), [x / 4 for x in f])
    ntk = rt.rope_plan(64, scaling="ntk", factor=4.0, **kw).freq.numpy()
    assert ntk[0] == 1.0 and abs(ntk[-1] * 4 / f[-1] - 1) < 1e-13
    yarn = rt.rope_plan(64, scaling="yarn", factor=4.0, original=4096, **kw)
    turns = [4096 * x / (2 * math.pi) for x in f]
    for x, n, y in zip(f, turns, yarn.freq.numpy()):
        want = x if n > 32 else (x / 4 if n < 1 else x / 4 + (x - x / 4) * (n - 1) / 31)
        assert abs(y / want - 1) < 1e-13
    assert yarn.amplitude == 0.1 * math.log(4.0) + 1
    three = rt.rope_plan(64, widths=(16, 24, 24), **kw)
    assert three.axis.tolist() == [0] * 8 + [1] * 12 + [2] * 12 and three.freq[8] == 1.0 and three.rotated == 64


@pytest.mark.parametrize("name", sorted(synth.WORKLOADS))
def test_grids(name):
    wl = synth.WORKLOADS[name]
    at, plan = schedule.grid_rope(wl, device="cpu")
    assert plan.rotated == wl.D and at.shape[0] == wl.T and not at[:wl.n_text].any()
    if plan.axes > 1:
        assert at.shape == (wl.T, plan.axes) and len({tuple(x) for x in at[wl.n_text:].tolist()}) == wl.T - wl.n_text
        assert at.amax(0).tolist() == [wl.frames - 1, wl.grid_h - 1, wl.grid_w - 1][3 - plan.axes:]
