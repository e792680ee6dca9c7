"""Gradients of dense and sparse attention against the 64-bit oracle, element by element inside the bounds that the
roundings of P, dS and the result allow (oracle/gradients.py), with the forward call's own output and statistics."""

import numpy as np
import pytest

import paper_2505_22918_amd as rt
from oracle import gradients as og
from paper_2505_22918_amd import synth
from parity import f64, to_dev, to_np

pytestmark = pytest.mark.gpu


def _inputs(B, H, T, D, seed, scale=1.0):
    rng = np.random.default_rng(seed)
    bits = [synth.f32_to_bf16_bits(rng.standard_normal((B, H, T, D), dtype=np.float32) * s)
            for s in (scale, 1.0, 1.0, 1.0)]
    return [to_dev(b) for b in bits], [f64(b) for b in bits]


def _masks(n, n_masks, keep, seed, column=None, unkept=None):
    """CSR of n_masks random masks with the diagonal, `column` kept by every row, and `unkept` by none but the first."""
    rng = np.random.default_rng(seed)
    row_ptr, col = [], []
    at = 0
    for _ in range(n_masks):
        row_ptr.append(at)
        for r in range(n):
            k = set(rng.choice(n, size=min(n, rng.integers(1, keep + 1)), replace=False).tolist()) | {r}
            if column is not None:
                k.add(column)
            if unkept is not None:
                k.discard(unkept)
                k = k or {0}
            col += sorted(k)
            at += len(k)
            row_ptr.append(at)
    return np.array(row_ptr), np.array(col)


def _check(got, ref, tol, what):
    assert np.isfinite(got).all(), f"{what}: not finite"
    err = np.abs(got - ref)
    worst = np.unravel_index(np.argmax(err / tol), err.shape)
    assert (err <= tol).all(), f"{what}: off {err[worst]:.3e} at {worst}, {tol[worst]:.3e} allowed"


def _compare(host, stats, grads, kept_of=None, w=None):
    q, k, v, d_o = host
    o, m, l = (to_np(x) for x in stats)
    grads = [to_np(g) for g in grads]
    B, H = q.shape[:2]
    for b in range(B):
        for h in range(H):
            a = (q[b, h], k[b, h], v[b, h], o[b, h], m[b, h], l[b, h], d_o[b, h],
                 None if kept_of is None else kept_of(b, h), None if w is None else w[b, h])
            ref, tol = og.head_backward(*a), og.head_tolerances(*a)
            for name, g, r, t in zip(("dq", "dk", "dv"), grads, ref, tol):
                _check(g[b, h], r, t, f"{name} of head {b},{h}")


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 129, 255, 257, 300, 700])
def test_full(gpu, D, T):
    print(f"[full backward] T={T} D={D}", flush=True)
    B, H = (2, 3) if T < 100 else (1, 2)
    dev, host = _inputs(B, H, T, D, 10 * T + D)
    stats = rt.attn_full(*dev[:3])
    _compare(host, stats, rt.attn_full_backward(*dev[:3], *stats, dev[3]))


@pytest.mark.parametrize("scale", [0.0, 4.0, 30.0])
def test_full_with_flat_and_peaked_rows(gpu, scale):
    dev, host = _inputs(1, 2, 190, 64, 3, scale)
    stats = rt.attn_full(*dev[:3])
    _compare(host, stats, rt.attn_full_backward(*dev[:3], *stats, dev[3]))


def test_full_long(gpu):
    dev, host = _inputs(1, 1, 2100, 72, 4)
    stats = rt.attn_full(*dev[:3])
    _compare(host, stats, rt.attn_full_backward(*dev[:3], *stats, dev[3]))


@pytest.mark.parametrize("H,T,D", [(1, 705, 64), (1, 1027, 72), (2, 1500, 64), (3, 1290, 72), (2, 2003, 72)])
def test_full_few_heads(gpu, H, T, D):
    """Few tiles: workgroups share a tile's walk, and the parts are added in order."""
    dev, host = _inputs(1, H, T, D, T)
    stats = rt.attn_full(*dev[:3])
    out = rt.attn_full_backward(*dev[:3], *stats, dev[3])
    _compare(host, stats, out)
    assert all((x == y).all() for x, y in zip(out, rt.attn_full_backward(*dev[:3], *stats, dev[3])))


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("T,masks,ratio", [(1, 1, False), (33, 1, True), (64, 1, False), (65, "H", True),
                                           (200, "BH", False), (300, 1, True), (517, "H", False), (900, "BH", True)])
def test_sparse(gpu, D, block, T, masks, ratio):
    print(f"[sparse backward] T={T} D={D} block={block} masks={masks} ratio={ratio}", flush=True)
    import torch

    B, H = 2, 3
    n = -(-T // block)
    n_masks = {1: 1, "H": H, "BH": B * H}[masks]
    rp, ci = _masks(n, n_masks, 4, T + block, column=n // 2)
    mask = rt.BlockMask.from_csr(rp, ci, block, n_masks=n_masks)
    dev, host = _inputs(B, H, T, D, T + D + block)
    stats = rt.attn_sparse(*dev[:3], mask)
    rho = w = None
    if ratio:
        rng = np.random.default_rng(T)
        r = rng.uniform(0.0, 1.0, (B, H, T)).astype(np.float32)
        r[0, 0, :3] = [0.0, 1.0, 0.75][:min(3, T)]
        rho = torch.from_numpy(r).cuda()
        ramped = (r + np.float32(0.25)).astype(np.float64)
        w = np.minimum(ramped, 1.0)
    out = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask, rho=rho, rho_delta=0.25)
    rows = rp.reshape(n_masks, n + 1)
    _compare(host, stats, out[:3],
             lambda b, h: og.token_mask(rows[{1: 0, "H": h, "BH": b * H + h}[masks]], ci, block, T), w)
    if ratio:
        o = to_np(stats[0])
        delta = (host[3] * o).sum(-1)
        ref = np.where(ramped <= 1.0, delta, 0.0)
        tol = (D + 8) * og.HALF_F32 * (np.abs(host[3]) * np.abs(o)).sum(-1) + og.TINY
        assert (np.abs(to_np(out[3]) - ref) <= tol).all()


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("block,T,masks", [(32, 3300, 1), (32, 3211, 2), (32, 3130, 4), (64, 6211, 1)])
def test_lists_that_are_split(gpu, D, block, T, masks):
    """A key block that every query block keeps: its list is walked in parts, which are joined."""
    print(f"[sparse backward, split] T={T} D={D} block={block} masks={masks}", flush=True)
    B, H = (1, 1) if masks == 1 else (2, 2)
    n = -(-T // block)
    rp, ci = _masks(n, masks, 3, T, column=n - 1)
    mask = rt.BlockMask.from_csr(rp, ci, block, n_masks=masks)
    # the plan behind the entries: one split list to a mask
    plan = mask.transposed().col_idx[-(-len(ci) // 4) * 4:].cpu().numpy().reshape(-1, 4)
    more = (len(plan) - masks * n) // 2
    assert sorted(x // n for x in plan[masks * n + more:, 0] if x >= 0) == list(range(masks))
    dev, host = _inputs(B, H, T, D, T + D + block)
    stats = rt.attn_sparse(*dev[:3], mask)
    out = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    rows = rp.reshape(masks, n + 1)
    _compare(host, stats, out, lambda b, h: og.token_mask(rows[{1: 0, 2: h, 4: b * H + h}[masks]], ci, block, T))


@pytest.mark.parametrize("block", [32, 64])
def test_a_key_block_that_no_query_keeps_gets_zero(gpu, block):
    T = 5 * block - 7
    rp, ci = _masks(5, 1, 2, 1, unkept=3)
    mask = rt.BlockMask.from_csr(rp, ci, block)
    dev, _ = _inputs(1, 2, T, 64, 9)
    stats = rt.attn_sparse(*dev[:3], mask)
    _, dk, dv = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    for g in (dk, dv):
        assert (g[:, :, 3 * block:4 * block] == 0).all()
        assert (g[:, :, 2 * block:3 * block] != 0).any()


def test_a_query_block_that_keeps_no_key_adds_nothing(gpu):
    import torch

    T, block = 256, 64
    dev, host = _inputs(1, 2, T, 64, 11)
    # not checked on the host: rows 0 and 2 are empty
    mask = rt.BlockMask(torch.tensor([0, 0, 2, 2, 4], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, 1, 1, 3], dtype=torch.int32, device="cuda"), block, 4, 4)
    o, m, l = rt.attn_sparse(*dev[:3], mask)
    dq, dk, dv = rt.attn_sparse_backward(*dev[:3], o, m, l, dev[3], mask)
    keep = np.r_[64:128, 192:256]
    assert (dq[:, :, :64] == 0).all() and (dq[:, :, 128:192] == 0).all()
    kept = og.token_mask([0, 0, 2, 2, 4], [0, 1, 1, 3], block, T)
    for h in range(2):
        a = [x[0, h] for x in host]
        on, mn, ln = (to_np(x)[0, h] for x in (o, m, l))
        # the empty rows out of the sums
        args = (a[0][keep], a[1], a[2], on[keep], mn[keep], ln[keep], a[3][keep], kept[keep])
        p = np.where(args[7], np.exp(args[0] @ a[1].T / 8 - args[4][:, None]) / args[5][:, None], 0)
        ds = p * (args[6] @ a[2].T - (args[6] * args[3]).sum(1)[:, None])
        # the sums' own error: a rounding of P or dS and one of the result, each term at its size
        for got, ref, size in ((dk, ds.T @ args[0] / 8, np.abs(ds).T @ np.abs(args[0]) / 8),
                               (dv, p.T @ args[6], p.T @ np.abs(args[6]))):
            assert (np.abs(to_np(got)[0, h] - ref) <= 2.5 * og.HALF_BF16 * size + 1e-5).all()


def test_row_past_the_factor_and_shared_entries_are_nan(gpu):
    import torch

    dev, _ = _inputs(1, 2, 128, 64, 12)
    mask = rt.BlockMask.from_csr([0, 1, 2], [0, 1], 64)
    stats = rt.attn_sparse(*dev[:3], mask)
    rho = torch.full((1, 2, 128), 0.5, device="cuda")
    rho[0, 0, 70] = 0.1
    dq, dk, dv, _ = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask, rho=rho, rho_delta=-0.25)
    assert torch.isnan(dq[0, 0, 70]).all() and torch.isfinite(dq[0, 0, :64]).all() and torch.isfinite(dq[0, 1]).all()
    assert torch.isnan(dv[0, 0, 64:]).all() and torch.isfinite(dv[0, 0, :64]).all()
    # two masks over the same entries: from_csr makes room, a mask made by hand does not
    rp, ci = [0, 1, 2, 0, 1, 2], [0, 1]
    shared = rt.BlockMask.from_csr(rp, ci, 64, n_masks=2)
    one = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    two = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], shared)
    assert all(torch.equal(x, y) for x, y in zip(one, two))
    raw = rt.BlockMask(shared.row_ptr, shared.col_idx, 64, 2, 2, 2)
    dq, dk, dv = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], raw)
    assert torch.equal(dq, one[0]) and torch.isnan(dk).all() and torch.isnan(dv).all()


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("block", [32, 64])
def test_a_row_that_is_not_finite_stays_in_its_blocks(gpu, D, block):
    """Of a block-diagonal mask, blocks beside the one with a NaN or an infinity keep their bits."""
    import torch

    T = 4 * block - 5
    mask = rt.BlockMask.from_csr(np.arange(5), np.arange(4), block)
    dev, _ = _inputs(1, 2, T, D, 13)
    stats = rt.attn_sparse(*dev[:3], mask)
    clean = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    for which, value in ((0, float("nan")), (1, float("inf")), (2, float("nan")), (3, float("inf"))):
        bad = [x.clone() for x in dev]
        bad[which][0, 0, block + 3, D - 1] = value
        got = rt.attn_sparse_backward(*bad[:3], *stats, bad[3], mask)
        for g, c in zip(got, clean):
            g, c = g.clone(), c.clone()
            g[0, 0, block:2 * block] = 0
            c[0, 0, block:2 * block] = 0
            assert torch.equal(g, c), which


def test_transposed_mask(gpu):
    for n, n_masks, keep in ((1, 1, 1), (5, 3, 2), (70, 2, 9), (300, 1, 40), (640, 2, 3), (641, 2, 3), (900, 1, 60)):
        rp, ci = _masks(n, n_masks, keep, n)
        t = rt.BlockMask.from_csr(rp, ci, 64, n_masks=n_masks).transposed()
        got_rp, got_ci = t.row_ptr.cpu().numpy().reshape(n_masks, n + 1), t.col_idx.cpu().numpy()
        rows = rp.reshape(n_masks, n + 1)
        at = 0
        for m in range(n_masks):
            for kb in range(n):
                ref = [r for r in range(n) if kb in ci[rows[m, r]:rows[m, r + 1]]]
                assert got_rp[m, kb] == at
                assert got_ci[at:at + len(ref)].tolist() == ref
                at += len(ref)
            assert got_rp[m, n] == at


@pytest.mark.parametrize("n,n_masks,keep", [(40, 2, 3), (97, 1, 2), (120, 3, 2), (300, 2, 60), (640, 1, 2), (700, 2, 3)])
def test_the_plan_covers_every_list_once(gpu, n, n_masks, keep):
    """Behind the entries: first parts, further parts, records of the split lists, whose parts are numbered in order."""
    rp, ci = _masks(n, n_masks, keep, n, column=n // 3)
    t = rt.BlockMask.from_csr(rp, ci, 64, n_masks=n_masks).transposed()
    plan = t.col_idx[-(-len(ci) // 4) * 4:].cpu().numpy().reshape(-1, 4)
    rows = t.row_ptr.cpu().numpy().reshape(n_masks, n + 1)
    more = (len(plan) - n_masks * n) // 2
    first, further, records = plan[:n_masks * n], plan[n_masks * n:n_masks * n + more], plan[n_masks * n + more:]
    further = [tuple(x) for x in further if x[0] >= 0]
    records = {x[0]: tuple(x[1:3]) for x in records if x[0] >= 0}
    slots = []
    for i, (row, at, count, slot) in enumerate(first):
        b, e = rows[i // n, i % n], rows[i // n, i % n + 1]
        parts = [(at, count, slot)] + [x[1:] for x in further if x[0] == i]
        assert row == i and [x[0] for x in parts] == sorted(x[0] for x in parts)
        assert b == at and sum(x[1] for x in parts) == e - b
        assert all(x[0] + x[1] == y[0] for x, y in zip(parts, parts[1:]))
        if len(parts) == 1:
            assert slot == -1 and i not in records
        else:
            assert records[i] == (slot, len(parts)) and [x[2] for x in parts] == list(range(slot, slot + len(parts)))
            slots += [x[2] for x in parts]
    assert len(slots) == len(set(slots)) and all(0 <= x < 2 * more for x in slots)
    assert len(records) == (n_masks if n > 96 and keep < 20 else 0) or keep >= 20


@pytest.mark.parametrize("D,block,n,H,masks", [(64, 32, 101, 160, 1), (72, 64, 101, 150, 1), (64, 64, 101, 96, 96),
                                               (72, 32, 101, 100, 200), (64, 32, 41, 500, 1)])
def test_parts_that_are_taken_together(gpu, D, block, n, H, masks):
    """Many heads: a workgroup takes two and more parts of a list together, or a list whole.  Some heads of them against
    the oracle."""
    B = 2 if masks > 1 else 1
    T = n * block - 5
    rp, ci = _masks(n, masks, 3, D + H, column=n - 2)
    kept = B * H * len(ci) // masks
    assert kept // 1536 >= 2 * 16, "a call that folds its parts"
    mask = rt.BlockMask.from_csr(rp, ci, block, n_masks=masks)
    dev, host = _inputs(B, H, T, D, D + block)
    stats = rt.attn_sparse(*dev[:3], mask)
    out = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    rows = rp.reshape(masks, n + 1)
    for b, h in ((0, 0), (B - 1, H // 2), (B - 1, H - 1)):
        one = lambda x: x[b:b + 1, h:h + 1]  # noqa: E731
        row = rows[0 if masks == 1 else (h if masks == H else b * H + h)]
        _compare([one(x) for x in host], [one(x) for x in stats], [one(x) for x in out],
                 lambda *_: og.token_mask(row, ci, block, T))


def test_equal_calls_give_equal_bits(gpu):
    import torch

    dev, _ = _inputs(2, 3, 1000, 64, 14)
    rp, ci = _masks(16, 1, 4, 2, column=0)
    mask = rt.BlockMask.from_csr(rp, ci, 64)
    for fwd, bwd in ((lambda: rt.attn_full(*dev[:3]), lambda s: rt.attn_full_backward(*dev[:3], *s, dev[3])),
                     (lambda: rt.attn_sparse(*dev[:3], mask),
                      lambda s: rt.attn_sparse_backward(*dev[:3], *s, dev[3], mask))):
        s = fwd()
        first = bwd(s)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(first, bwd(s)))


@pytest.mark.parametrize("D", [64, 72])
@pytest.mark.parametrize("T", [37, 200, 530])
def test_full_many_heads(gpu, D, T):
    """More workgroups than CUs: another kernel than few heads take."""
    B, H = 8, 40
    dev, host = _inputs(B, H, T, D, T + D)
    stats = rt.attn_full(*dev[:3])
    out = rt.attn_full_backward(*dev[:3], *stats, dev[3])
    pick = [(0, 0), (3, 17), (7, 39)]
    sub = lambda t: np.stack([to_np(t[b, h]) for b, h in pick])[None]  # noqa: E731
    q, k, v, d_o = (np.stack([x[b, h] for b, h in pick])[None] for x in host)
    o, m, l = (sub(x) for x in stats)
    for i in range(len(pick)):
        a = (q[0, i], k[0, i], v[0, i], o[0, i], m[0, i], l[0, i], d_o[0, i])
        for name, g, r, t in zip(("dq", "dk", "dv"), out, og.head_backward(*a), og.head_tolerances(*a)):
            _check(sub(g)[0, i], r, t, f"{name} of head {pick[i]}")


def test_largest_head(gpu):
    """One head of the longest sequence whose offsets the kernels hold, block-diagonal: each block is an attention of its
    own.  (131072 blocks: the transpose by searches; offsets of 2^30 bytes.)"""
    import torch

    T, D, block = 1 << 23, 64, 64
    n = T // block
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, d_o = (torch.randn(1, 1, T, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    at = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    mask = rt.BlockMask(at, at[:n].clone(), block, n, n)
    print("[sparse backward] largest head", flush=True)
    o, m, l = rt.attn_sparse(q, k, v, mask)
    out = rt.attn_sparse_backward(q, k, v, o, m, l, d_o, mask)
    torch.cuda.synchronize()
    for b in (0, 1, n // 2, n - 2, n - 1):
        part = lambda t: to_np(t[0, 0, b * block:(b + 1) * block])  # noqa: E731
        a = tuple(part(t) for t in (q, k, v, o, m, l, d_o))
        for name, x, r, t in zip(("dq", "dk", "dv"), out, og.head_backward(*a), og.head_tolerances(*a)):
            _check(part(x), r, t, f"{name} of block {b}")


def test_a_transpose_of_anything_stays_in_its_arrays(gpu):
    """The gradient call does not trust what the transpose holds: entries, parts and blocks out of range are left out."""
    import torch

    from paper_2505_22918_amd import _lib

    T, n = 256, 4
    dev, _ = _inputs(1, 2, T, 64, 15)
    mask = rt.BlockMask.from_csr(np.arange(0, 2 * n + 1, 2), [0, 1, 0, 1, 2, 3, 2, 3], 64)
    stats = rt.attn_sparse(*dev[:3], mask)
    want = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
    t = mask.transposed()
    for junk in (0, 7, 1 << 20, 0x7fffffff, -1, -0x80000000):
        t.col_idx.fill_(junk)
        dq, dk, dv = rt.attn_sparse_backward(*dev[:3], *stats, dev[3], mask)
        torch.cuda.synchronize()
        assert torch.equal(dq, want[0]) and dk.shape == dv.shape, junk
    assert _lib.load().rt_last_error() == b""
