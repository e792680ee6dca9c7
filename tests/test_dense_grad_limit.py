"""Dense gradients at the most heads that one launch takes."""

import pytest

from paper_2505_22918_amd import _lib

AT = [0x7F0000000000 + i * (1 << 38) for i in range(12)]  # never dereferenced
MOST = 8 * ((1 << 20) - 1)  # tiles of one launch of 2^32 threads, in whole eights: both halves of 256 threads each


@pytest.mark.parametrize("heads", [MOST + 1, MOST + 7])
def test_one_more_is_refused_on_the_host(heads):
    lib = _lib.load()
    for T in (1, 64):
        assert lib.rt_attn_full_backward(*AT[:7], _lib.RtDims(1, heads, T, 64), *AT[7:11], 1 << 36, None) == _lib.RT_EINVAL
        assert "too many" in lib.rt_last_error().decode()


@pytest.mark.gpu
def test_the_most(gpu):
    """Heads of one token: P is 1, so dv is d_o, and o is v, so dS is what the two sums' roundings leave of 0."""
    import torch

    import paper_2505_22918_amd as rt

    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, d_o = (torch.randn(1, MOST, 1, 64, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    m = (q[..., 0, :].float() * k[..., 0, :].float()).sum(-1, keepdim=True) / 8
    print("[full backward] the most heads", flush=True)
    dq, dk, dv = rt.attn_full_backward(q, k, v, v, m, torch.ones_like(m), d_o)
    torch.cuda.synchronize()
    assert torch.equal(dv, d_o)
    # two sums of 64 products, each off by at most 64 roundings of 2^-24
    most = (d_o.float() * v.float()).abs().sum(-1, keepdim=True) * (2 * 66 * 2.0 ** -24 / 8)
    for got, other in ((dq, k), (dk, q)):
        assert bool((got.float().abs() <= most * other.float().abs() * (1 + 2.0 ** -7) + 1e-30).all())
