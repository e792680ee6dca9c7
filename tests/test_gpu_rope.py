"""Rotary positions against the fp64 oracle: layouts, parts of the head, axes, types, strides, positions far out; in
place, in graphs, on other streams; refusals."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import heads as oh

pytestmark = pytest.mark.gpu

HALF_STEP = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}


def _x(shape, dtype, seed=0):
    import torch

    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(getattr(torch, dtype)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _check(y, x, positions, plan, inverse=False):
    axis = None if plan.axis is None else plan.axis.cpu().numpy()
    ref = oh.rope(_np(x), positions.cpu().numpy(), plan.freq.cpu().numpy(), axis, plan.amplitude, plan.layout, inverse)
    largest = float(positions.double().abs().max() * plan.freq.max())
    tol = oh.rope_tolerance(_np(x), ref, plan.freq.numel(), HALF_STEP[str(x.dtype).split(".")[1]], plan.amplitude, plan.layout,
                            largest)
    err = np.abs(_np(y) - ref)
    assert y.dtype is x.dtype and y.shape == x.shape
    worst = float((err / np.maximum(tol, 1e-300)).max(initial=0.0))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("shape,rotated", [((1, 1, 1, 2), 2), ((2, 3, 5, 64), 64), ((1, 5, 33, 72), 72), ((2, 2, 7, 72), 48),
                                           ((1, 30, 19, 64), 24), ((1, 9, 300, 128), 10), ((3, 1, 2, 67), 64), ((1, 6, 4, 18), 6)])
def test_layouts_and_widths(gpu, dtype, layout, shape, rotated):
    import torch

    x = _x(shape, dtype)
    plan = rt.rope_plan(rotated, base=100.0, layout=layout)
    pos = torch.arange(shape[2], device="cuda") + 11
    _check(rt.rope(x, pos, plan), x, pos, plan)
    _check(rt.rope_backward(x, pos, plan), x, pos, plan, inverse=True)


@pytest.mark.parametrize("kind", ["int32", "int64", "float32"])
@pytest.mark.parametrize("start", [0, 4095, 1000003, 16777000])
def test_positions_far_out(gpu, kind, start):
    import torch

    x = _x((2, 3, 40, 64), "float32", 1)
    pos = (torch.arange(80).reshape(2, 40) + start).to(getattr(torch, kind)).cuda()
    for plan in (rt.rope_plan(64), rt.rope_plan(64, base=500000.0, layout="half")):
        _check(rt.rope(x, pos, plan), x, pos, plan)
        _check(rt.rope(x, pos[1], plan), x, pos[1], plan)
    if kind == "int64":
        far = pos + (1 << 33)
        _check(rt.rope(x, far, plan), x, far, plan)
        _check(rt.rope(x, -far, plan), x, -far, plan)


def test_fractions_of_positions_and_no_position(gpu):
    import torch

    x = _x((1, 4, 50, 64), "bfloat16", 2)
    plan = rt.rope_plan(64)
    pos = torch.linspace(0, 29, 50).cuda()
    _check(rt.rope(x, pos, plan), x, pos, plan)
    assert torch.equal(rt.rope(x, torch.zeros(50, dtype=torch.int32, device="cuda"), plan), x)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_axes_of_a_grid_behind_text(gpu, layout):
    import torch

    t = torch.arange(3 * 4 * 5)
    grid = torch.stack([t // 20, t // 5 % 4, t % 5], -1)
    pos = torch.cat([torch.zeros((7, 3), dtype=torch.int64), grid]).cuda()
    x = _x((2, 6, 67, 64), "bfloat16", 3)
    plan = rt.rope_plan(64, widths=(16, 24, 24), layout=layout)
    y = rt.rope(x, pos, plan)
    _check(y, x, pos, plan)
    assert torch.equal(y[:, :, :7], x[:, :, :7])
    both = torch.stack([pos, pos.flip(0).contiguous()])
    _check(rt.rope(x, both, plan), x, both, plan)


def test_amplitude(gpu):
    import torch

    x = _x((1, 2, 9, 64), "float32", 4)
    plan = rt.rope_plan(48, scaling="yarn", factor=8.0, original=16)
    pos = torch.arange(9, device="cuda") * 100
    y = rt.rope(x, pos, plan)
    _check(y, x, pos, plan)
    assert torch.equal(y[..., 48:], x[..., 48:])


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_strides(gpu, layout):
    import torch

    plan = rt.rope_plan(64, layout=layout)
    packed = _x((2, 31, 3, 5, 64), "bfloat16", 5)
    pos = torch.arange(31, device="cuda")
    qk = packed[:, :, :2].flatten(2, 3).transpose(1, 2)
    assert qk.data_ptr() == packed.data_ptr()
    y = rt.rope(qk, pos, plan)
    assert y.is_contiguous()
    _check(y, qk, pos, plan)
    # into a packed gradient, whose other part stays as it is
    grad = torch.full_like(packed, 7.0)
    out = grad[:, :, :2].flatten(2, 3).transpose(1, 2)
    assert rt.rope_backward(y, pos, plan, out=out) is out
    _check(out, y, pos, plan, inverse=True)
    assert bool((grad[:, :, 2] == 7).all())
    # rows that start on no 16 or 8 bytes, every second token, an expanded head
    odd = _x((2 * 3 * 31 * 67 + 1,), "bfloat16", 6)[1:].view(2, 3, 31, 67)[..., :64]
    _check(rt.rope(odd, pos, plan), odd, pos, plan)
    half = packed[:, ::2, 0].transpose(1, 2)
    _check(rt.rope(half, pos[:16].contiguous(), plan), half, pos[:16], plan)
    one = _x((2, 1, 31, 64), "bfloat16", 7).expand(2, 9, 31, 64)
    _check(rt.rope(one, pos, plan), one, pos, plan)
    four = _x((1, 2, 31, 68), "bfloat16", 8)[..., 4:]
    _check(rt.rope(four, pos, plan), four, pos, plan)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("D,rotated", [(64, 64), (72, 72), (67, 40), (128, 96)])
def test_in_place(gpu, layout, D, rotated):
    import torch

    plan = rt.rope_plan(rotated, layout=layout)
    x = _x((2, 13, 21, D), "bfloat16", 9)
    pos = torch.arange(21, device="cuda")
    want = rt.rope(x, pos, plan)
    y = x.clone()
    assert rt.rope(y, pos, plan, out=y) is y
    assert torch.equal(y, want)


def test_gradient_is_the_transpose(gpu):
    import torch

    plan = rt.rope_plan(56, scaling="yarn", factor=4.0, original=64, layout="half")
    x, d_y = _x((1, 3, 17, 72), "float32", 10), _x((1, 3, 17, 72), "float32", 11)
    pos = torch.arange(17, device="cuda") * 31
    a = (rt.rope(x, pos, plan).double() * d_y.double()).sum()
    b = (x.double() * rt.rope_backward(d_y, pos, plan).double()).sum()
    # 6 + 1 roundings of 32 bits a product of 1.2 amplitude, at most, and both sums
    assert abs(a - b) <= 2 * 7 * 2.0 ** -24 * 2 * plan.amplitude * float((x.abs().max() * d_y.double().abs()).sum())


def test_non_finite_values_stay_in_their_pair(gpu):
    import torch

    plan = rt.rope_plan(64)
    x = _x((1, 1, 8, 72), "bfloat16", 12)
    pos = torch.arange(8, device="cuda")
    want = rt.rope(x, pos, plan)
    x[0, 0, 3, 10], x[0, 0, 5, 70] = float("nan"), float("inf")
    got = rt.rope(x, pos, plan)
    bad = ~torch.isfinite(got)
    assert bad.nonzero().tolist() == [[0, 0, 3, 10], [0, 0, 3, 11], [0, 0, 5, 70]]
    assert torch.equal(got[~bad], want[~bad])


def test_empty_calls(gpu):
    import torch

    plan = rt.rope_plan(64)
    for shape in ((0, 2, 3, 64), (2, 0, 3, 64), (2, 2, 0, 64)):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        assert rt.rope(x, torch.arange(shape[2], device="cuda"), plan).shape == shape


def test_many_heads_of_few_tokens_and_few_of_many(gpu):
    import torch

    plan = rt.rope_plan(72, layout="half")
    for shape in ((1, 1000, 1, 72), (1, 1, 5000, 72), (1, 3, 1, 72)):
        x = _x(shape, "bfloat16", 13)
        pos = torch.arange(shape[2], device="cuda") + 5
        _check(rt.rope(x, pos, plan), x, pos, plan)


def test_graph_and_streams(gpu):
    import torch

    plan = rt.rope_plan(64)
    x, pos = _x((2, 8, 50, 64), "bfloat16", 14), torch.arange(50, device="cuda")
    y = torch.empty_like(x)
    rt.rope(x, pos, plan, out=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rt.rope(x, pos, plan, out=y)
    for seed in range(3):
        x.copy_(_x(x.shape, "bfloat16", 20 + seed))
        pos += 100
        y.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, rt.rope(x, pos, plan))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = rt.rope(x, pos, plan)
    side.synchronize()
    assert torch.equal(z, y)


def test_refusals(gpu):
    import torch

    plan, x, pos = rt.rope_plan(64), _x((2, 3, 5, 64), "bfloat16"), torch.arange(5, device="cuda")
    bad = [
        (x.cpu(), pos, plan), (x, pos.cpu(), plan), (x, pos[:4], plan), (x, pos.half(), plan), (x, pos, None),
        (x[0], pos, plan), (x.double(), pos, plan), (x.transpose(2, 3), pos, plan), (x, torch.arange(10, device="cuda")[::2], plan),
        (x, pos.expand(2, 5), plan), (x, pos.expand(3, 5).contiguous(), plan), (x, pos[:, None].contiguous(), plan),
        (x, pos, rt.rope_plan(64, device="cpu")), (x, pos, rt.RopePlan(plan.freq.float())), (x, pos, rt.RopePlan(plan.freq, axes=2)),
        (x, pos, rt.RopePlan(plan.freq, layout="other")), (x, pos, rt.RopePlan(plan.freq, plan.freq, 2)),
        (x, pos, rt.rope_plan(64, widths=(32, 32))),
    ]
    for a in bad:
        for fn in (rt.rope, rt.rope_backward):
            with pytest.raises(ValueError):
                fn(*a)
    for out in (x.float(), x[:, :2], x.cpu(), x.transpose(0, 2), 3):
        with pytest.raises(ValueError):
            rt.rope(x, pos, plan, out=out)
    big = _x((2, 3, 6, 64), "bfloat16")
    for out, of in ((big[:, :, 1:], big[:, :, :5]), (big[:, :1, :5].expand(2, 3, 5, 64), x)):
        with pytest.raises(rt.RettentionError) as e:
            rt.rope(of, pos, plan, out=out)
        assert e.value.status == 1
    with pytest.raises(rt.RettentionError):
        rt.rope(x, pos, rt.rope_plan(72))  # more than the row has
    for kw in (dict(rotated=63), dict(rotated=0), dict(rotated=64, widths=(32, 30)), dict(rotated=64, widths=(63, 1)),
               dict(rotated=64, base=0.0), dict(rotated=64, factor=-1.0), dict(rotated=64, layout="x"),
               dict(rotated=64, scaling="x"), dict(rotated=64, scaling="yarn", factor=2.0), dict(rotated=64, base=float("nan"))):
        with pytest.raises(ValueError):
            rt.rope_plan(**kw)
