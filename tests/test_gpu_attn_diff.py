"""Differential attention and its gradients against the fp64 oracle: sizes from one row up, other numbers of keys than
of queries, padded keys, split walks, one weight or one for each head; graphs, streams, refusals; the layer's calls
together."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import heads as oh

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


def _inputs(B, H, Tq, Tk, D, seed=0, scale=1.0):
    import torch

    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    q, k, v, do = (x.bfloat16().cuda() for x in (n(B, 2 * H, Tq, D) * scale, n(B, 2 * H, Tk, D), n(B, H, Tk, 2 * D), n(B, H, Tq, 2 * D)))
    return q, k, v, do, (0.5 + 0.2 * n(H)).cuda()


def _within(got, ref, tol, what):
    assert got.shape == ref.shape, what
    with np.errstate(invalid="ignore"):
        err = np.abs(np.where(np.isinf(ref), 0.0, got - ref))
    assert np.array_equal(np.isinf(got), np.isinf(ref)), what
    assert np.all(err <= tol), (what, float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))


def _check_forward(out, q, k, v, lam, lens=None):
    o, o2, m, l = (_np(x) for x in out)
    B, H, Tk = v.shape[:3]
    q, k, v, lam = _np(q), _np(k), _np(v), np.broadcast_to(_np(lam), (H,))
    for b in range(B):
        for h in range(H):
            maps = slice(2 * h, 2 * h + 2)
            ref, tol = oh.forward(q[b, maps], k[b, maps], v[b, h], lam[h], Tk if lens is None else lens[b])
            for x, r, t, name in zip((o[b, h], o2[b, h], m[b, maps], l[b, maps]), ref, tol, ("o", "o2", "m", "l")):
                _within(x, r, t, (name, b, h))


def _check_backward(got, q, k, v, out, do, lam, lens=None):
    dq, dk, dv, dlam = (_np(x) for x in got)
    B, H, Tk = v.shape[:3]
    o, o2, m, l = (_np(x) for x in out)
    q, k, v, do, ln = _np(q), _np(k), _np(v), _np(do), np.broadcast_to(_np(lam), (H,))
    sums, tols = np.zeros(H), np.zeros(H)
    for b in range(B):
        for h in range(H):
            maps = slice(2 * h, 2 * h + 2)
            ref, tol = oh.backward(q[b, maps], k[b, maps], v[b, h], o[b, h], o2[b, h], m[b, maps], l[b, maps], do[b, h], ln[h],
                                   Tk if lens is None else lens[b])
            for x, r, t, name in zip((dq[b, maps], dk[b, maps], dv[b, h]), ref, tol, ("dq", "dk", "dv")):
                _within(x, r, t, (name, b, h))
            sums[h] += ref[3]
            tols[h] += tol[3]
    if lam.numel() != H:
        sums, tols = sums.sum(), tols.sum()
    assert got[3].shape == lam.shape
    _within(dlam.reshape(-1), np.reshape(sums, -1), np.reshape(tols, -1), "dlam")


def _lens(lens):
    import torch

    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


SIZES = [(1, 1, 1, 1), (1, 1, 1, 2), (2, 3, 1, 300), (1, 2, 15, 2000), (1, 1, 16, 33), (2, 1, 17, 700), (2, 1, 32, 32), (1, 2, 33, 31), (1, 1, 64, 65), (2, 2, 127, 63), (1, 1, 128, 200), (1, 3, 129, 129),
         (1, 1, 300, 1), (1, 1, 5, 700), (2, 3, 100, 70), (1, 1, 128, 128), (1, 2, 90, 500), (1, 2, 700, 5), (1, 1, 257, 1100),
         # waves of four on 128 rows, whole and in parts; gradients in parts of either side's walk, and of both
         (1, 40, 300, 130), (1, 40, 200, 1500), (1, 1, 33, 1000), (1, 1, 33, 700), (1, 1, 129, 700), (1, 1, 513, 64), (1, 20, 33, 1000),
         (3, 12, 513, 64), (1, 8, 1100, 1000)]


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("B,H,Tq,Tk", SIZES)
def test_sizes(gpu, B, H, Tq, Tk, D):
    print(f"[diff] B={B} H={H} Tq={Tq} Tk={Tk} D={D}", flush=True)
    q, k, v, do, lam = _inputs(B, H, Tq, Tk, D, Tq + Tk)
    out = rt.attn_diff(q, k, v, lam)
    _check_forward(out, q, k, v, lam)
    import torch

    assert torch.equal(rt.attn_diff(q, k, v, lam, stats=False), out[0])
    got = rt.attn_diff_backward(q, k, v, *out, do, lam)
    _check_backward(got, q, k, v, out, do, lam)


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("Tq,Tk,lens", [(40, 100, [100, 37, 0, 1]), (1, 500, [500, 33, 0, 256]), (16, 3000, [3000, 1, 0, 1700]), (9, 130, [130, 97, 0, 64]), (200, 130, [64, 128, 129, 0]),
                                        (300, 700, [700, 5, 0, 333]), (7, 65, [-3, 99, 64, 65])])
def test_padded_keys(gpu, Tq, Tk, lens, D):
    import torch

    print(f"[diff] Tq={Tq} Tk={Tk} lens={lens} D={D}", flush=True)
    q, k, v, do, lam = _inputs(4, 2, Tq, Tk, D, 7)
    used = [min(max(n, 0), Tk) for n in lens]
    # what lies past a sample's keys is not used, whatever it holds
    bad_k, bad_v = k.clone(), v.clone()
    for b, n in enumerate(used):
        bad_k[b, :, n:], bad_v[b, :, n:] = float("nan"), float("inf")
    lens = _lens(lens)
    out = rt.attn_diff(q, k, v, lam, k_lens=lens)
    _check_forward(out, q, k, v, lam, used)
    for x, y in zip(out, rt.attn_diff(q, bad_k, bad_v, lam, k_lens=lens)):
        assert torch.equal(x, y)
    got = rt.attn_diff_backward(q, k, v, *out, do, lam, k_lens=lens)
    _check_backward(got, q, k, v, out, do, lam, used)
    for x, y in zip(got, rt.attn_diff_backward(q, bad_k, bad_v, *out, do, lam, k_lens=lens)):
        assert torch.equal(x, y)
    for b, n in enumerate(used):
        assert not got[1][b, :, n:].any() and not got[2][b, :, n:].any()


# samples are taken by their numbers of keys up to 64 of them, in whatever order they lie
@pytest.mark.parametrize("B,H,Tq,Tk,D", [(64, 1, 40, 70, 64), (65, 1, 40, 70, 72), (3, 5, 260, 300, 72), (2, 3, 700, 50, 64), (5, 1, 33, 1500, 64), (9, 2, 129, 257, 72)])
def test_padded_order(gpu, B, H, Tq, Tk, D):
    import torch

    print(f"[diff] order of samples B={B} H={H} Tq={Tq} Tk={Tk} D={D}", flush=True)
    q, k, v, do, lam = _inputs(B, H, Tq, Tk, D, 13)
    g = torch.Generator().manual_seed(13)
    used = [int(x) for x in torch.randint(-3, Tk + 4, (B,), generator=g)]
    used[-1], used[0] = Tk, used[B // 2]  # the longest last, two alike
    lens, clamped = _lens(used), [min(max(n, 0), Tk) for n in used]
    out = rt.attn_diff(q, k, v, lam, k_lens=lens)
    _check_forward(out, q, k, v, lam, clamped)
    got = rt.attn_diff_backward(q, k, v, *out, do, lam, k_lens=lens)
    _check_backward(got, q, k, v, out, do, lam, clamped)
    to = torch.randperm(B, generator=g).cuda()
    moved = rt.attn_diff(q[to], k[to], v[to], lam, k_lens=lens[to])
    for x, y in zip(moved, out):
        assert torch.equal(x, y[to])
    for x, y in zip(rt.attn_diff_backward(q[to], k[to], v[to], *moved, do[to], lam, k_lens=lens[to])[:3], got):
        assert torch.equal(x, y[to])


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("Tq", [5, 70, 300])
def test_running_max_moves(gpu, Tq, D):
    # scores that rise by hundreds from tile to tile, fall again, and lie far below zero
    q, k, v, do, lam = _inputs(1, 1, Tq, 400, D, 9)
    import torch

    ramp = torch.linspace(-40, 60, 400, device="cuda")
    ramp[200:300] = -50
    q[..., 0], k[..., 0] = 4.0, ramp.bfloat16()
    k[0, 1, :, 0] = ramp.flip(0).bfloat16()
    out = rt.attn_diff(q, k, v, lam)
    _check_forward(out, q, k, v, lam)
    got = rt.attn_diff_backward(q, k, v, *out, do, lam)
    _check_backward(got, q, k, v, out, do, lam)


@pytest.mark.parametrize("shape", [(), (1,)])
def test_one_weight_for_all_heads(gpu, shape):
    import torch

    q, k, v, do, _ = _inputs(2, 3, 150, 90, 64, 11)
    lam = torch.full(shape, 0.31, device="cuda")
    out = rt.attn_diff(q, k, v, lam)
    _check_forward(out, q, k, v, lam)
    _check_backward(rt.attn_diff_backward(q, k, v, *out, do, lam), q, k, v, out, do, lam)


def test_weight_of_zero_is_plain_attention(gpu):
    import torch

    q, k, v, _, _ = _inputs(1, 2, 130, 130, 64, 12)
    o, o2, m, l = rt.attn_diff(q, k, v, torch.zeros(2, device="cuda"))
    for i in range(2):
        for half in range(2):
            o_f, m_f, l_f = rt.attn_full(q[:, i::2].contiguous(), k[:, i::2].contiguous(), v[..., 64 * half:64 * half + 64].contiguous())
            mine = (o, o2)[i][..., 64 * half:64 * half + 64]
            # both round probabilities and the result to bf16 (half a step each)
            assert float((mine.double() - o_f.double()).abs().max()) <= 2 * 2 * 2.0 ** -8 * float(v.abs().max())
            assert torch.equal(m[:, i::2], m_f)
            assert float((l[:, i::2] / l_f - 1).abs().max()) <= 2 * (130 + 8) * 2.0 ** -24


def test_gradients_are_differences(gpu):
    # of the fp32 sums behind a forward output in bf16: steps as large as the result's rounding allows
    import torch

    q, k, v, do, lam = _inputs(1, 1, 64, 96, 64, 13)
    out = rt.attn_diff(q, k, v, lam)
    dq, dk, dv, dlam = rt.attn_diff_backward(q, k, v, *out, do, lam)

    def value(q, k, v, lam):
        o = rt.attn_diff(q, k, v, lam, stats=False)
        return float((o.double() * do.double()).sum())

    g = torch.Generator().manual_seed(1)
    for i, (x, grad) in enumerate(zip((q, k, v, lam), (dq, dk, dv, dlam))):
        step = (torch.randn(x.shape, generator=g).cuda() * 0.25).to(x.dtype)
        up, down = (x.float() + step.float()).to(x.dtype), (x.float() - step.float()).to(x.dtype)
        args = [q, k, v, lam]
        args[i] = up
        a = value(*args)
        args[i] = down
        b = value(*args)
        want = float(((up.double() - down.double()) * grad.double()).sum())
        # each output is rounded twice by half a step; a third-order term of the size of the step's square
        noise = 4 * 2.0 ** -8 * float((out[0].double() * do.double()).square().sum().sqrt()) + 0.25 ** 2 * abs(want)
        scale = float(((up.double() - down.double()) * grad.double()).square().sum().sqrt())
        assert abs((a - b) - want) <= noise + 0.25 * scale + 0.5, (i, a - b, want)


def test_equal_calls_give_equal_bits(gpu):
    import torch

    for B, H, Tq, Tk, D in ((1, 2, 500, 900, 64), (2, 1, 1, 3000, 72), (1, 1, 2000, 40, 72)):
        q, k, v, do, lam = _inputs(B, H, Tq, Tk, D, 14)
        out = rt.attn_diff(q, k, v, lam)
        got = rt.attn_diff_backward(q, k, v, *out, do, lam)
        for _ in range(3):
            again = rt.attn_diff(q, k, v, lam)
            assert all(torch.equal(x, y) for x, y in zip(out, again))
            assert all(torch.equal(x, y) for x, y in zip(got, rt.attn_diff_backward(q, k, v, *again, do, lam)))


@pytest.mark.parametrize("B,H,Tq,Tk", [(0, 2, 3, 4), (2, 0, 3, 4), (2, 2, 0, 4), (2, 2, 3, 0), (1, 1, 0, 0)])
def test_empty_calls(gpu, B, H, Tq, Tk):
    q, k, v, do, lam = _inputs(B, H, Tq, Tk, 64)
    out = rt.attn_diff(q, k, v, lam)
    got = rt.attn_diff_backward(q, k, v, *out, do, lam)
    assert not any(x.any() for x in (out[0], out[1], out[3], *got))
    assert bool((out[2] == float("-inf")).all())
    import torch

    one = torch.tensor(0.5, device="cuda")
    out = rt.attn_diff(q, k, v, one)
    assert float(rt.attn_diff_backward(q, k, v, *out, do, one)[3]) == 0.0


def test_given_outputs_and_their_neighbours(gpu):
    import torch

    q, k, v, do, lam = _inputs(2, 1, 45, 77, 72, 15)
    want = rt.attn_diff(q, k, v, lam)
    grads = rt.attn_diff_backward(q, k, v, *want, do, lam)

    def framed(like):
        whole = torch.full((like.numel() + 512,), 3.0, dtype=like.dtype, device="cuda")
        return whole, whole[256:256 + like.numel()].view(like.shape)

    whole, o = framed(want[0])
    assert rt.attn_diff(q, k, v, lam, out=o)[0] is o
    assert torch.equal(o, want[0]) and bool((whole[:256] == 3).all()) and bool((whole[256 + o.numel():] == 3).all())
    frames = [framed(x) for x in grads[:3]]
    got = rt.attn_diff_backward(q, k, v, *want, do, lam, out=[x for _, x in frames])
    for (whole, x), g, y in zip(frames, grads, got):
        assert y is x and torch.equal(x, g) and bool((whole[:256] == 3).all()) and bool((whole[256 + x.numel():] == 3).all())


def test_non_finite_rows_stay_in_their_row(gpu):
    import torch

    for D, Tq, bad in ((64, 70, (5, 40)), (72, 70, (5, 40)), (64, 11, (3, 9)), (72, 11, (3, 9)), (72, 900, (300, 301))):
        q, k, v, _, lam = _inputs(1, 1, Tq, 90, D, 16)
        want = rt.attn_diff(q, k, v, lam)
        q[0, 0, bad[0], 3], q[0, 1, bad[1], 60] = float("nan"), float("inf")
        got = rt.attn_diff(q, k, v, lam)
        rows = [r for r in range(Tq) if r not in bad]
        for x, y in zip(got, want):
            assert torch.equal(x[:, :, rows], y[:, :, rows])
        assert bool(torch.isnan(got[0][0, 0, list(bad)]).all())


def test_graphs_share_inputs_not_workspaces(gpu):
    import torch

    for Tq, Tk in ((1, 2000), (300, 700)):
        q, k, v, do, lam = _inputs(2, 2, Tq, Tk, 64, 17)
        lens = _lens([Tk, Tk // 2])

        def step():
            out = rt.attn_diff(q, k, v, lam, k_lens=lens)
            return out + rt.attn_diff_backward(q, k, v, *out, do, lam, k_lens=lens)

        step()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = step()
            graphs.append((g, out))
        for seed in range(3):
            n = _inputs(2, 2, Tq, Tk, 64, 30 + seed)
            for x, y in zip((q, k, v, do, lam), n):
                x.copy_(y)
            lens.copy_(_lens([Tk - seed, 1 + 400 * seed]))
            for g, _ in graphs:
                g.replay()
            torch.cuda.synchronize()
            for _, out in graphs:
                assert all(torch.equal(x, y) for x, y in zip(out, step()))


def test_streams(gpu):
    import torch

    q, k, v, do, lam = _inputs(1, 2, 200, 1500, 64, 18)
    want = rt.attn_diff(q, k, v, lam)
    grads = rt.attn_diff_backward(q, k, v, *want, do, lam)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                out = rt.attn_diff(q, k, v, lam)
                results.append((out, rt.attn_diff_backward(q, k, v, *out, do, lam)))
    torch.cuda.synchronize()
    for out, got in results:
        assert all(torch.equal(x, y) for x, y in zip(out, want)) and all(torch.equal(x, y) for x, y in zip(got, grads))


def test_refusals(gpu):
    import torch

    q, k, v, do, lam = _inputs(1, 2, 8, 9, 64)
    out = rt.attn_diff(q, k, v, lam)
    bad = [dict(q=q.cpu()), dict(k=k.float()), dict(v=v[..., :64]), dict(q=q[:, :3].contiguous()), dict(k=k[:, :2].contiguous()),
           dict(q=q.transpose(2, 3)), dict(v=v.transpose(0, 1)), dict(lam=lam.double()), dict(lam=lam[:1].expand(3)),
           dict(lam=torch.zeros(3, device="cuda")), dict(lam=0.5), dict(lam=lam.cpu()), dict(k_lens=_lens([1, 2])),
           dict(k_lens=_lens([1]).long()), dict(k_lens=_lens([1]).cpu()), dict(k_lens=5)]
    for kw in bad:
        a = dict(q=q, k=k, v=v, lam=lam, **{x: y for x, y in kw.items() if x == "k_lens"})
        a.update(kw)
        with pytest.raises(ValueError):
            rt.attn_diff(**a)
        with pytest.raises(ValueError):
            rt.attn_diff_backward(a["q"], a["k"], a["v"], *out, do, a["lam"], k_lens=a.get("k_lens"))
    for i in range(5):
        args = [*out, do]
        args[i] = args[i][:, :, :7]
        with pytest.raises(ValueError):
            rt.attn_diff_backward(q, k, v, *args, lam)
    with pytest.raises(ValueError):
        rt.attn_diff(q, k, v, lam, out=out[0][:, :1])
    with pytest.raises(ValueError):
        rt.attn_diff_backward(q, k, v, *out, do, lam, out=(q, k))
    with pytest.raises(rt.RettentionError) as e:
        rt.attn_diff_backward(q, k, v, *out, do, lam, out=(q, torch.empty_like(k), torch.empty_like(v)))
    assert e.value.status == 1
    wide = [torch.zeros((1, n, 4, d), dtype=torch.bfloat16, device="cuda") for n, d in ((2, 80), (2, 80), (1, 160))]
    with pytest.raises(rt.RettentionError) as e:
        rt.attn_diff(*wide, lam[:1])
    assert e.value.status == 2


@pytest.mark.parametrize("D", [64, 72])
def test_a_layer_forward_and_back(gpu, D):
    """Packed projection -> norm of queries and keys -> rotary positions -> differential attention -> norm of the heads,
    and the gradients back to the projection and the weights, against the same chain in 64 bits by autograd."""
    import torch

    B, H, T = 2, 2, 130
    g = torch.Generator().manual_seed(21)
    qk = torch.randn((B, T, 2, 2 * H, D), generator=g).bfloat16().cuda()
    v = torch.randn((B, H, T, 2 * D), generator=g).bfloat16().cuda()
    d_y = torch.randn((B, H, T, 2 * D), generator=g).bfloat16().cuda()
    wq, wk, wo = (1 + 0.1 * torch.randn(n, generator=g).cuda() for n in (D, D, 2 * D))
    lam = (0.5 + 0.1 * torch.randn(H, generator=g)).cuda()
    pos, lens = torch.arange(T, device="cuda") + 50, _lens([T, 77])
    plan = rt.rope_plan(D, layout="half")

    x = qk.permute(2, 0, 3, 1, 4)
    normed = [rt.layer_norm(x[i], w, eps=1e-6, stats=True) for i, w in enumerate((wq, wk))]
    q, k = (rt.rope(y, pos, plan) for y, _, _ in normed)
    out = rt.attn_diff(q, k, v, lam, k_lens=lens)
    y, mean, rstd = rt.layer_norm(out[0], wo, stats=True)
    d_o, d_wo, _ = rt.layer_norm_backward(d_y, out[0], mean, rstd, wo, bias=False)
    dq, dk, dv, dlam = rt.attn_diff_backward(q, k, v, *out, d_o, lam, k_lens=lens)
    d_qk = torch.zeros_like(qk)
    d_x = d_qk.permute(2, 0, 3, 1, 4)
    d_w = []
    for i, (grad, (_, mu, rs), w) in enumerate(zip((dq, dk), normed, (wq, wk))):
        rt.rope_backward(grad, pos, plan, out=grad)
        d_w.append(rt.layer_norm_backward(grad, x[i], mu, rs, w, bias=False, out=d_x[i])[1])

    # 64 bits, on the CPU
    leaf = [t.double().cpu().requires_grad_() for t in (qk, v, wq, wk, wo, lam)]
    Q, V, WQ, WK, WO, L = leaf
    f = plan.freq.cpu()
    ang = pos.cpu().double()[:, None] * f
    norm = lambda t, w, e: torch.nn.functional.layer_norm(t, t.shape[-1:], eps=e) * w  # noqa: E731

    def turn(t):
        a, b = t.chunk(2, -1)
        return torch.cat([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1)

    X = Q.permute(2, 0, 3, 1, 4)
    S = turn(norm(X[0], WQ, 1e-6)) @ turn(norm(X[1], WK, 1e-6)).transpose(2, 3) / D ** 0.5
    S = S.masked_fill(torch.arange(T) >= lens.cpu()[:, None, None, None], -np.inf)
    A = S.softmax(-1).unflatten(1, (H, 2))
    Y = norm((A[:, :, 0] - L[:, None, None] * A[:, :, 1]) @ V, WO, 1e-5)
    (Y * d_y.double().cpu()).sum().backward()
    # a chain of roundings to bf16: of x's norm, the rotation, P, o, the norm and back again, 12 of half a step at most on
    # any path, taken together as independent ones of 2^-8 / sqrt(3) each; the output's norm divides by a spread that
    # is about sqrt(1 + lam^2) / sqrt(keys) of v's
    limit = 4 * (12 / 3) ** 0.5 * 2.0 ** -8
    for got, ref in ((y, Y.detach()), (d_qk, Q.grad), (dv, V.grad), (d_wo, WO.grad), (d_w[0], WQ.grad), (d_w[1], WK.grad), (dlam, L.grad)):
        err = (got.double().cpu() - ref).norm() / ref.norm()
        assert float(err) <= limit, float(err)
    assert not d_qk[1, 77:, 1].any()
