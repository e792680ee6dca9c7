"""Rotary positions and differential attention past 32-bit offsets, and at full length against 64 bits on the GPU."""

import pytest

import paper_2505_22918_amd as rt

pytestmark = pytest.mark.gpu


def _bf16(*shape):
    import torch

    return torch.randn(shape, device="cuda", dtype=torch.bfloat16)


def test_a_long_cache_past_4_gib(gpu):
    import torch

    H, Tk = 40, 500_000  # 5.1 GB of keys, as much of values
    torch.manual_seed(1)
    q, do, k, v = _bf16(1, 2 * H, 1, 64), _bf16(1, H, 1, 128), _bf16(1, 2 * H, Tk, 64), _bf16(1, H, Tk, 128)
    lam = torch.full((H,), 0.4, device="cuda")
    out = rt.attn_diff(q, k, v, lam)
    grads = rt.attn_diff_backward(q, k, v, *out, do, lam)
    for h in (0, H - 1):
        two = slice(2 * h, 2 * h + 2)
        qh, kh, vh = q[:, two].contiguous(), k[:, two].contiguous(), v[:, h:h + 1].contiguous()
        S = (qh.double() @ kh.double().transpose(2, 3))[0, :, 0] / 8
        P = S.softmax(-1)
        o = torch.stack([P[i] @ vh[0, 0].double() for i in range(2)])
        # probabilities and the result rounded by half a step of bf16, independent over 500000 keys: bounded by the norm
        size = (P.square() @ vh[0, 0].double().square()).sqrt()
        want = o[0] - 0.4 * o[1]
        assert bool(((out[0][0, h, 0].double() - want).abs() <= 2.0 ** -8 * (want.abs() + 6 * (size[0] + 0.4 * size[1]))).all())
        mine = [x[:, two].contiguous() if i >= 2 else x[:, h:h + 1].contiguous() for i, x in enumerate(out)]
        alone = rt.attn_diff_backward(qh, kh, vh, *mine, do[:, h:h + 1].contiguous(), lam[:1])
        # one query: a key's gradient is one product, however the walks are shared out
        assert torch.equal(grads[1][:, two], alone[1]) and torch.equal(grads[2][:, h:h + 1], alone[2])


def test_rows_past_4_gib_are_turned(gpu):
    import torch

    x, pos, plan = _bf16(1, 40, 1_000_000, 64), torch.arange(1_000_000, device="cuda"), rt.rope_plan(64)
    y = rt.rope(x, pos, plan)
    for h in (0, 39):
        assert torch.equal(y[:, h:h + 1], rt.rope(x[:, h:h + 1], pos, plan))
    assert torch.equal(y[:, :, 999_000:], rt.rope(x[:, :, 999_000:], pos[999_000:], plan))


@pytest.mark.parametrize("D,T", [(64, 17776), (72, 16384)])
def test_a_head_at_full_length(gpu, D, T):
    import torch

    torch.manual_seed(2)
    q, k, v, do = _bf16(1, 2, T, D), _bf16(1, 2, T, D), _bf16(1, 1, T, 2 * D), _bf16(1, 1, T, 2 * D)
    lam = torch.tensor([0.6], device="cuda")
    o, o2, m, l = out = rt.attn_diff(q, k, v, lam)
    got = rt.attn_diff_backward(q, k, v, *out, do, lam)
    Q, K, V, G = (x[0].double() for x in (q, k, v, do))
    A = [torch.softmax(Q[i] @ K[i].t() / D ** 0.5, -1) for i in range(2)]
    O = [a @ V[0] for a in A]
    pull = G[0] @ V[0].t()
    inner2 = (G[0] * o2[0, 0].double()).sum(-1)
    inner1 = (G[0] * o[0, 0].double()).sum(-1) + 0.6 * inner2
    S = A[0] * (pull - inner1[:, None]), A[1] * (pull - inner2[:, None]) * -0.6
    want = {"o": O[0] - 0.6 * O[1], "o2": O[1], "dq": torch.stack([S[i] @ K[i] for i in range(2)]) / D ** 0.5,
            "dk": torch.stack([S[i].t() @ Q[i] for i in range(2)]) / D ** 0.5, "dv": (A[0] - 0.6 * A[1]).t() @ G[0]}
    have = {"o": o[0, 0], "o2": o2[0, 0], "dq": got[0][0], "dk": got[1][0], "dv": got[2][0, 0]}
    for n, w in want.items():
        # operands of the products and the results rounded by up to half a step each: sqrt(2) 2^-8 / sqrt(3) as
        # independent errors, 2^-8 at most is asked
        err = float((have[n].double() - w).norm() / w.norm())
        assert err <= 2.0 ** -8, (n, err)
    # sums of T and 2 D products in 32 bits behind them, delta's in the 128 and more of a row
    z = (Q[0] @ K[0].t()).div_(D ** 0.5)
    assert float((m[0, 0].double() - z.amax(-1)).abs().max()) <= (D + 8) * 2.0 ** -24 * 40
    assert float((l[0, 0].double() / (z - m[0, 0].double()[:, None]).exp().sum(-1) - 1).abs().max()) <= (T + 64) * 2.0 ** -24
    assert abs(float(got[3]) + float(inner2.sum())) <= (2 * D + 8) * 2.0 ** -24 * float((G[0] * o2[0, 0].double()).abs().sum())
