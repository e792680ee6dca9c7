"""The multi-step driver with the layer norm of queries and keys in front of attention: the same steps made by hand."""

import json

import pytest

import paper_2505_22918_amd as rt
from paper_2505_22918_amd import schedule

pytestmark = pytest.mark.gpu


def test_driver_norms_queries_and_keys(gpu):
    import torch

    T = 300
    g = torch.Generator().manual_seed(1)
    qkv = tuple((torch.randn(1, 2, T, 64, generator=g) * s + 0.5).bfloat16().cuda() for s in (3.0, 2.0, 1.0))
    norm = tuple((1 + 0.1 * torch.randn(64, generator=g).cuda(), 0.1 * torch.randn(64, generator=g).cuda())
                 for _ in range(2))
    n = -(-T // 64)
    mask = rt.BlockMask.from_csr(list(range(0, 2 * n + 1, 2)), [c for r in range(n) for c in sorted({r, (r + 1) % n})], 64)
    drift = lambda prev, t: tuple((x.float() * 0.97).bfloat16() for x in prev)  # noqa: E731
    _, outs = schedule.run(mask, qkv, 6, 2, 3, 0.01, 0.0, diagnose=False, evolve=drift, qk_norm=norm)
    cache, cur = rt.StatCache(mask, 2, 3, 0.01), qkv
    for t, out in enumerate(outs):
        if t:
            cur = drift(cur, t)
        q, k = (rt.layer_norm(x, w, b, eps=1e-6) for x, (w, b) in zip(cur, norm))
        assert torch.equal(out, cache.attend(q, k, cur[2], t)), t
    plain = schedule.run(mask, qkv, 1, 2, 3, 0.0, 0.0, diagnose=False)[1][0]
    assert not torch.equal(plain, outs[0])


def test_command_line(gpu, capsys):
    assert schedule.main(["--workload", "tiny", "--steps", "3", "--full-steps", "1", "--qk-norm"]) == 0
    lines = [json.loads(x) for x in capsys.readouterr().out.strip().splitlines()]
    assert len(lines) == 4 and lines[-1]["summary"]["reshape_steps"] == 2
