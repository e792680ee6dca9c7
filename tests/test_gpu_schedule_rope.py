"""The multi-step driver with rotary positions of queries and keys in front of attention: the same steps made by hand."""

import json

import pytest

import paper_2505_22918_amd as rt
from paper_2505_22918_amd import schedule

pytestmark = pytest.mark.gpu


def test_driver_turns_queries_and_keys(gpu):
    import torch

    T = 300
    g = torch.Generator().manual_seed(1)
    qkv = tuple(torch.randn(1, 2, T, 64, generator=g).bfloat16().cuda() for _ in range(3))
    one = (torch.ones(64, device="cuda"), torch.zeros(64, device="cuda"))
    at, plan = torch.arange(T, device="cuda"), rt.rope_plan(64)
    n = -(-T // 64)
    mask = rt.BlockMask.from_csr(list(range(0, 2 * n + 1, 2)), [c for r in range(n) for c in sorted({r, (r + 1) % n})], 64)
    drift = lambda prev, t: tuple((x.float() * 0.97).bfloat16() for x in prev)  # noqa: E731
    for norm in (None, (one, one)):
        _, outs = schedule.run(mask, qkv, 6, 2, 3, 0.01, 0.0, diagnose=False, evolve=drift, qk_norm=norm, qk_rope=(at, plan))
        cache, cur = rt.StatCache(mask, 2, 3, 0.01), qkv
        for t, out in enumerate(outs):
            if t:
                cur = drift(cur, t)
            q, k = cur[:2] if norm is None else (rt.layer_norm(x, *w, eps=1e-6) for x, w in zip(cur, norm))
            assert torch.equal(out, cache.attend(rt.rope(q, at, plan), rt.rope(k, at, plan), cur[2], t)), t


@pytest.mark.parametrize("extra", [[], ["--qk-norm"]])
def test_command_line(gpu, capsys, extra):
    assert schedule.main(["--workload", "tiny", "--steps", "3", "--full-steps", "1", "--qk-rope", *extra]) == 0
    lines = [json.loads(x) for x in capsys.readouterr().out.strip().splitlines()]
    assert len(lines) == 4 and lines[-1]["summary"]["reshape_steps"] == 2
