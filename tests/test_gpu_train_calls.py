"""The training calls as a program makes them: a whole layer's step against 64-bit autograd, in captured graphs whose
inputs change between replays, on other streams, with outputs that the caller owns, and refused arguments."""

import ctypes

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import gradients as og

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8  # half a step of bf16


def _mask(n, keep, seed, block=64, n_masks=1):
    rng = np.random.default_rng(seed)
    rp, ci = [], []
    for _ in range(n_masks):
        rp.append(len(ci))
        for r in range(n):
            ci += sorted(set(rng.choice(n, size=min(n, keep), replace=False).tolist()) | {r})
            rp.append(len(ci))
    return rt.BlockMask.from_csr(rp, ci, block, n_masks=n_masks), rp, ci


def _bf16(*shape, seed=0, scale=1.0):
    import torch

    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).bfloat16().cuda()


# ---- one step of a layer ------------------------------------------------------------------


def _layer(p, x, kept, block, rho, resid, delta):
    """The step's forward in 64 bits by elementary operations: norm, projection, head norms, attention over the kept
    blocks (all where kept is None) and the reshape, output projection."""
    import torch

    B, N, C = x.shape
    H, D = p["H"], p["D"]

    def norm(t, w, b):
        t = t - t.mean(-1, keepdim=True)
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w + b

    h = norm(x, p["w0"][:, None], p["b0"][:, None])
    qkv = (h @ p["wqkv"]).reshape(B, N, 3, H, D).permute(2, 0, 3, 1, 4)
    q, k, v = norm(qkv[0], p["wq"], p["bq"]), norm(qkv[1], p["wk"], p["bk"]), qkv[2]
    s = q @ k.transpose(-1, -2) / D ** 0.5
    if kept is not None:
        s = s.masked_fill(~kept, -float("inf"))
    o = torch.softmax(s, -1) @ v
    if rho is not None:
        o = torch.clamp(rho + delta, max=1.0)[..., None] * o + resid
    return o.permute(0, 2, 1, 3).reshape(B, N, H * D) @ p["wo"]


@pytest.mark.parametrize("D,sparse", [(64, False), (64, True), (72, False), (72, True)])
def test_a_layer_of_the_training_step(gpu, D, sparse):
    """Forward and backward of norm, projection, head norms, attention and the reshape from the library's calls (and
    torch's products) against autograd in 64 bits on the same bf16 inputs.  The path rounds to bf16 about a dozen times
    in a row (norm, projection, head norms, scores' inputs, P, output, and their gradients): 12 times half a step of
    each value, 2-norm against 2-norm, where single rounding errors add up in squares."""
    import torch

    torch.manual_seed(3)
    B, N, H = 2, 330, 3
    C = H * D
    f = lambda *s, scale=1.0: (torch.randn(s, dtype=torch.float64) * scale)  # noqa: E731
    p = dict(H=H, D=D, w0=1 + 0.1 * f(B, C), b0=0.1 * f(B, C), wqkv=f(C, 3 * C, scale=C ** -0.5), wq=1 + 0.1 * f(D),
             bq=0.1 * f(D), wk=1 + 0.1 * f(D), bk=0.1 * f(D), wo=f(C, C, scale=C ** -0.5))
    x, dy = f(B, N, C), f(B, N, C)
    rho, resid = torch.rand(B, H, N, dtype=torch.float64) * 0.9, f(B, H, N, D, scale=0.3)
    names = ["w0", "b0", "wqkv", "wq", "bq", "wk", "bk", "wo"]
    half = lambda t: t.bfloat16().cuda()  # noqa: E731
    single = lambda t: t.float().cuda()  # noqa: E731
    X, dY, Wqkv, Wo, R, Rho = half(x), half(dy), half(p["wqkv"]), half(p["wo"]), half(resid), single(rho)
    W = {n: single(p[n]) for n in names if n not in ("wqkv", "wo")}
    mask, rp, ci = _mask(-(-N // 64), 2, 4)
    delta = 0.05

    # the library's step
    h, m0, r0 = rt.layer_norm(X, W["w0"], W["b0"], eps=1e-6, stats=True)
    qkv = (h.reshape(-1, C) @ Wqkv).reshape(B, N, 3, H, D)
    view = [qkv[:, :, i].transpose(1, 2) for i in range(3)]
    q, mq, rq = rt.layer_norm(view[0], W["wq"], W["bq"], eps=1e-6, stats=True)
    k, mk, rk = rt.layer_norm(view[1], W["wk"], W["bk"], eps=1e-6, stats=True)
    v = view[2].contiguous()
    if sparse:
        o, m, l = rt.attn_sparse(q, k, v, mask)
        out = rt.reshape_apply(o, Rho, R, rho_delta=delta)
    else:
        o, m, l = rt.attn_full(q, k, v)
        out = o
    flat = out.transpose(1, 2).reshape(-1, C)
    y = flat @ Wo
    d = {"wo": flat.t().contiguous() @ dY.reshape(-1, C)}
    d_out = (dY.reshape(-1, C) @ Wo.t().contiguous()).reshape(B, N, H, D).transpose(1, 2).contiguous()
    d_qkv = torch.empty_like(qkv)
    grads = [d_qkv[:, :, i].transpose(1, 2) for i in range(3)]
    if sparse:
        dq, dk, dv, d["rho"] = rt.attn_sparse_backward(q, k, v, o, m, l, d_out, mask, rho=Rho, rho_delta=delta)
        d["resid"] = d_out
    else:
        dq, dk, dv = rt.attn_full_backward(q, k, v, o, m, l, d_out)
    grads[2].copy_(dv)
    _, d["wq"], d["bq"] = rt.layer_norm_backward(dq, view[0], mq, rq, W["wq"], out=grads[0])
    _, d["wk"], d["bk"] = rt.layer_norm_backward(dk, view[1], mk, rk, W["wk"], out=grads[1])
    d["wqkv"] = h.reshape(-1, C).t().contiguous() @ d_qkv.reshape(-1, 3 * C)
    d_h = (d_qkv.reshape(-1, 3 * C) @ Wqkv.t().contiguous()).reshape(B, N, C)
    d["x"], d["w0"], d["b0"] = rt.layer_norm_backward(d_h, X, m0, r0, W["w0"])

    # and autograd's, of the values that the library was given
    p64 = {n: (t.double().cpu().requires_grad_() if torch.is_tensor(t) else t)
           for n, t in dict(p, **W, wqkv=Wqkv, wo=Wo).items()}
    x64, rho64, resid64 = (t.double().cpu().requires_grad_() for t in (X, Rho, R))
    kept = torch.from_numpy(og.token_mask(rp, ci, 64, N)) if sparse else None
    ref = _layer(p64, x64, kept, 64, rho64 if sparse else None, resid64, delta)
    ref.backward(dY.double().cpu())
    want = {n: p64[n].grad for n in names} | {"x": x64.grad}
    if sparse:
        want |= {"rho": rho64.grad, "resid": resid64.grad}
    assert float((y.reshape(B, N, C).double().cpu() - ref.detach()).norm() / ref.detach().norm()) <= 12 * HALF
    for n, r in want.items():
        got = d[n].double().cpu()
        if n == "bk":
            # A shift of all keys by one vector shifts a row's scores by one number, so this gradient, the sum of dK's
            # rows, is 0: sum_j dK_j = sum_i q_i sum_j dS_ij, and sum_j dS_ij = sum_j P_ij dP_ij - delta_i sum_j P_ij = 0.
            # What is left is the sum of the rows' roundings, which are measured against dK itself.
            assert float(r.norm()) <= 1e-9 and float(got.norm()) <= 12 * HALF * float(dk.double().norm())
            continue
        assert got.shape == r.shape and float((got - r).norm() / r.norm()) <= 12 * HALF, n


# ---- captured graphs ----------------------------------------------------------------------


def _capture(fn):
    import torch

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


@pytest.mark.parametrize("T", [300, 1100])
def test_gradients_replay(gpu, T):
    """Dense and sparse gradients in one graph; inputs change between the replays, with eager calls in between."""
    import torch

    q, k, v, d_o = (_bf16(1, 3, T, 64, seed=s) for s in range(4))
    mask, _, _ = _mask(-(-T // 64), 3, 5)
    rho = torch.rand(1, 3, T, device="cuda")
    stats, sparse = rt.attn_full(q, k, v), rt.attn_sparse(q, k, v, mask)
    outs = [torch.empty_like(q) for _ in range(6)]
    d_rho = {}

    def step():
        rt.attn_full_backward(q, k, v, *stats, d_o, out=outs[:3])
        d_rho["g"] = rt.attn_sparse_backward(q, k, v, *sparse, d_o, mask, rho=rho, rho_delta=0.1, out=outs[3:])[3]

    g = _capture(step)
    for i in range(4):
        for t in outs:
            t.zero_()
        d_o.mul_(-0.75)
        rho.mul_(0.9)
        torch.cuda.synchronize()
        eager = rt.attn_full_backward(q, k, v, *stats, d_o)
        eager += rt.attn_sparse_backward(q, k, v, *sparse, d_o, mask, rho=rho, rho_delta=0.1)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + [d_rho["g"]], eager)), f"replay {i}"


def test_a_mask_first_transposed_in_a_graph(gpu):
    """The transpose that a capture builds belongs to the graph: eager calls afterwards make their own."""
    import torch

    T = 500
    q, k, v, d_o = (_bf16(1, 2, T, 64, seed=s) for s in range(4))
    mask, rp, ci = _mask(8, 3, 6)
    stats = rt.attn_sparse(q, k, v, mask)
    want = rt.attn_sparse_backward(q, k, v, *stats, d_o, rt.BlockMask.from_csr(rp, ci, 64))
    outs = [torch.empty_like(q) for _ in range(3)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rt.attn_sparse_backward(q, k, v, *stats, d_o, mask, out=outs)
    # before any replay: nothing of the capture may be used
    assert all(torch.equal(a, b) for a, b in zip(rt.attn_sparse_backward(q, k, v, *stats, d_o, mask), want))
    for _ in range(3):
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_a_run_time_mask_and_its_gradient_replay(gpu):
    """Mask from the step's Q and K, sparse attention over it and its gradients, captured together: the lists change
    with the inputs."""
    import torch

    T = 700
    q, k, v, d_o = (_bf16(1, 2, T, 64, seed=s) for s in range(4))
    outs = [torch.empty_like(q) for _ in range(3)]

    def step():
        mask = rt.dynamic_index(q, k, 64, 4)
        o, m, l = rt.attn_sparse(q, k, v, mask)
        return rt.attn_sparse_backward(q, k, v, o, m, l, d_o, mask, out=outs)

    g = _capture(step)
    for i in range(3):
        q.copy_(_bf16(1, 2, T, 64, seed=20 + i))
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), f"replay {i}"


def test_norms_replay(gpu):
    import torch

    x, dy = _bf16(2, 900, 64, seed=1), _bf16(2, 900, 64, seed=2)
    w, b = torch.rand(64, device="cuda"), torch.rand(64, device="cuda")
    res = {}

    def step():
        y, mean, rstd = rt.layer_norm(x, w, b, stats=True)
        res["all"] = (y, mean, rstd) + rt.layer_norm_backward(dy, x, mean, rstd, w)

    g = _capture(step)
    kept = res["all"]
    for i in range(4):
        x.mul_(0.5).add_(0.25)
        dy.mul_(-1.5)
        torch.cuda.synchronize()
        step()
        eager = [t.clone() for t in res["all"]]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager)), f"replay {i}"


# ---- streams, owners, refusals ------------------------------------------------------------


def test_calls_run_on_the_current_stream(gpu):
    """Behind a wait on another stream the inputs are ready only there."""
    import torch

    T = 900
    q, k, v, d_o = (_bf16(1, 4, T, 72, seed=s) for s in range(4))
    mask, rp, ci = _mask(15, 3, 7)
    want = rt.attn_sparse_backward(q, k, v, *rt.attn_sparse(q, k, v, mask), d_o, mask)
    y, mean, rstd = rt.layer_norm(q, stats=True)
    dx = rt.layer_norm_backward(d_o, q, mean, rstd)[0]
    torch.cuda.synchronize()
    late = [torch.zeros_like(t) for t in (q, k, v, d_o)]
    fresh = rt.BlockMask.from_csr(rp, ci, 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(torch.ones(2048, 2048, device="cuda"), torch.ones(2048, 2048, device="cuda"))
        for a, b in zip(late, (q, k, v, d_o)):
            a.copy_(b)
        got = rt.attn_sparse_backward(*late[:3], *rt.attn_sparse(*late[:3], fresh), late[3], fresh)
        y2, mean2, rstd2 = rt.layer_norm(late[0], stats=True)
        dx2 = rt.layer_norm_backward(late[3], late[0], mean2, rstd2)[0]
    # the transpose made on that stream, used on this one without a synchronisation in between
    again = rt.attn_sparse_backward(q, k, v, *rt.attn_sparse(q, k, v, fresh), d_o, fresh)
    torch.cuda.synchronize()
    for a, b, c in zip(got, want, again):
        assert torch.equal(a, b) and torch.equal(c, b)
    assert torch.equal(y, y2) and torch.equal(dx, dx2)


def test_outputs_of_the_caller(gpu):
    import torch

    q, k, v, d_o = (_bf16(1, 2, 200, 64, seed=s) for s in range(4))
    stats = rt.attn_full(q, k, v)
    want = rt.attn_full_backward(q, k, v, *stats, d_o)
    # rows of one allocation, with guards around them that stay as they were
    buf = torch.full((5, 2, 200, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = (buf[1:2], buf[2:3], buf[3:4])
    got = rt.attn_full_backward(q, k, v, *stats, d_o, out=out)
    assert all(a is b for a, b in zip(got, out)) and all(torch.equal(a, b) for a, b in zip(got, want))
    assert (buf[0] == 3.0).all() and (buf[4] == 3.0).all()
    with pytest.raises(rt.RettentionError):
        rt.attn_full_backward(q, k, v, *stats, d_o, out=(buf[1:2], buf[1:2], buf[3:4]))
    with pytest.raises(rt.RettentionError):
        rt.attn_full_backward(q, k, v, *stats, d_o, out=(q, buf[1:2], buf[3:4]))


def test_binding_refusals(gpu):
    import torch

    q, k, v, d_o = (_bf16(1, 2, 128, 64, seed=s) for s in range(4))
    mask, _, _ = _mask(2, 1, 1)
    o, m, l = rt.attn_sparse(q, k, v, mask)
    rho = torch.rand(1, 2, 128, device="cuda")
    bad = [lambda: rt.attn_full_backward(q, k, v, o, m, l, d_o.float()),
           lambda: rt.attn_full_backward(q, k, v, o, m, l, d_o.cpu()),
           lambda: rt.attn_full_backward(q, k, v, o[:, :1], m, l, d_o),
           lambda: rt.attn_full_backward(q, k, v, o, m.double(), l, d_o),
           lambda: rt.attn_full_backward(q, k, v, o, m, l, d_o.transpose(1, 2)),
           lambda: rt.attn_full_backward(q, k, v, o, m, l, d_o, out=(q.clone(), k.clone())),
           lambda: rt.attn_sparse_backward(q, k, v, o, m, l, d_o, mask, rho=rho[:, :1]),
           lambda: rt.layer_norm(q.double()),
           lambda: rt.layer_norm(q.cpu()),
           lambda: rt.layer_norm(q.transpose(2, 3)),
           lambda: rt.layer_norm(q[0, 0, 0]),
           lambda: rt.layer_norm(q, torch.ones(63, device="cuda")),
           lambda: rt.layer_norm(q, torch.ones(64, device="cuda").half()),
           lambda: rt.layer_norm(q, torch.ones(64, device="cuda"), torch.ones(1, 64, device="cuda")),
           lambda: rt.layer_norm(q, torch.ones(64)),
           lambda: rt.layer_norm(q, out=torch.empty_like(q).float()),
           lambda: rt.layer_norm_backward(d_o.float(), q, m, l),
           lambda: rt.layer_norm_backward(d_o, q, m[..., :5], l)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted:", i)
    for call in (lambda: rt.layer_norm(q, eps=-1.0), lambda: rt.layer_norm(q, out=q),
                 lambda: rt.layer_norm(torch.zeros(2, 16400, device="cuda")),
                 lambda: rt.layer_norm(q, out=torch.empty(64, device="cuda").bfloat16().expand(1, 2, 128, 64)),
                 lambda: rt.attn_sparse_backward(q, k, v, o, m, l, d_o, mask, rho=rho, rho_delta=float("nan"))):
        with pytest.raises(rt.RettentionError):
            call()


def test_empty_batches(gpu):
    import torch

    q = torch.empty(0, 2, 128, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.empty(0, 2, 128, device="cuda")
    assert all(t.shape == q.shape for t in rt.attn_full_backward(q, q, q, q, s, s, q))
    mask, _, _ = _mask(2, 1, 1)
    out = rt.attn_sparse_backward(q, q, q, q, s, s, q, mask, rho=s)
    assert len(out) == 4 and out[3].shape == s.shape


def test_small_workspace_is_refused(gpu):
    from paper_2505_22918_amd import _lib

    q = _bf16(1, 1, 64, 64)
    x = [torch_ptr for torch_ptr in (q.data_ptr(),)]
    outs = [_bf16(1, 1, 64, 64, seed=9 + i) for i in range(4)]
    stat = _bf16(2, 64).float()
    need = ctypes.c_int64()
    dims = _lib.RtDims(1, 1, 64, 64)
    assert gpu.rt_attn_full_backward_workspace(dims, ctypes.byref(need)) == _lib.RT_OK
    ptrs = [t.data_ptr() for t in outs]
    assert gpu.rt_attn_full_backward(x[0], x[0], x[0], x[0], stat.data_ptr(), stat.data_ptr(), x[0], dims, *ptrs,
                                     need.value - 1, None) == _lib.RT_ECAPACITY
