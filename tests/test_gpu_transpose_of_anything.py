"""What a transpose holds is not trusted: with lists that are split, parts taken together and joined, any values in it
leave the gradient calls inside their arrays, and dq as it was."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from test_gpu_attn_backward import _inputs, _masks

pytestmark = pytest.mark.gpu


def _guarded(q):
    """Three outputs with a margin around each, and the margins."""
    import torch

    n, room = q.numel(), 1 << 16
    buf = torch.full((3, n + 2 * room), 3.0, dtype=q.dtype, device=q.device)
    return tuple(b[room:room + n].view(q.shape) for b in buf), [b[x] for b in buf for x in (slice(0, room), slice(room + n, None))]


@pytest.mark.parametrize("D,block,H,masks", [(64, 32, 3, 1), (72, 64, 4, 4), (64, 64, 2, 1), (64, 32, 160, 1)])
def test_any_values(gpu, D, block, H, masks):
    import torch

    n = 101
    T = n * block - 5
    rp, ci = _masks(n, masks, 3, D + H, column=n - 2)
    mask = rt.BlockMask.from_csr(rp, ci, block, n_masks=masks)
    dev, _ = _inputs(1, H, T, D, D + block)
    stats = rt.attn_sparse(*dev[:3], mask)
    want = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    t = mask.transposed()
    plan = t.col_idx[-(-len(ci) // 4) * 4:].view(-1, 4)
    assert bool((plan[masks * n:] >= 0).any()), "a list is split"
    good, good_rows = t.col_idx.clone(), t.row_ptr.clone()
    g = torch.Generator(device="cuda").manual_seed(H)
    big, small = (lambda like, m=m: torch.randint(-m, m, like.shape, generator=g, device="cuda", dtype=torch.int32)
                  for m in (0x7fffffff, 300))

    def plan_only(values):
        def fill():
            plan.copy_(values(plan))
        return fill

    def first_column_kept(values):  # items of blocks that are there, their entries and parts anything
        def fill():
            plan[:, 1:].copy_(values(plan[:, 1:]))
        return fill

    fills = [lambda: t.col_idx.fill_(5), lambda: t.col_idx.fill_(-1), lambda: t.col_idx.fill_(0x7fffffff),
             lambda: t.col_idx.copy_(big(t.col_idx)), lambda: t.col_idx.copy_(small(t.col_idx)),
             plan_only(big), plan_only(small), first_column_kept(big), first_column_kept(small),
             lambda: t.row_ptr.copy_(big(t.row_ptr)), lambda: t.row_ptr.copy_(small(t.row_ptr))]
    for i, fill in enumerate(fills):
        print(f"[transpose of anything] D={D} block={block} H={H} masks={masks} fill {i}", flush=True)
        t.col_idx.copy_(good)
        t.row_ptr.copy_(good_rows)
        fill()
        out, margins = _guarded(dev[0])
        rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask, out=out, transposed=t)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]), i
        assert all(bool((x == 3.0).all()) for x in margins), i
    t.col_idx.copy_(good)
    t.row_ptr.copy_(good_rows)
    assert all(torch.equal(a, b) for a, b in zip(rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask, transposed=t), want))


@pytest.mark.parametrize("n,n_masks,keep,column", [(97, 1, 60, 30), (300, 2, 60, 100), (120, 3, 2, 40), (700, 2, 40, 3)])
def test_records_of_split_lists(gpu, n, n_masks, keep, column):
    """Exactly the lists longer than twice the mean, and than 16, have a record, by their length in parts."""
    rp, ci = _masks(n, n_masks, keep, n, column=column)
    t = rt.BlockMask.from_csr(rp, ci, 64, n_masks=n_masks).transposed()
    plan = t.col_idx[-(-len(ci) // 4) * 4:].cpu().numpy().reshape(-1, 4)
    more = (len(plan) - n_masks * n) // 2
    rows = np.asarray(rp).reshape(n_masks, n + 1)
    seg = max(16, 2 * -(-len(ci) // (n_masks * n)))
    want = {}
    for m in range(n_masks):
        lists = np.bincount(ci[rows[m, 0]:rows[m, -1]], minlength=n)
        want.update({m * n + kb: -(-int(c) // seg) for kb, c in enumerate(lists) if c > seg})
    assert want and {int(x[0]): int(x[2]) for x in plan[n_masks * n + more:] if x[0] >= 0} == want
