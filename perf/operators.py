"""The training operators of an attention layer, as they are measured: gradients of attention, and the layer norm.

  full_backward    gradients of dense attention, from its output and row statistics
  sparse_backward  gradients of attention over a block mask, with or without the reshape (the gradient of
                   min(1, rho + rho_delta) * SparseAttention(Q, K, V) + R for Q, K, V and rho)
  norm             layer norm of rows, in the layout that the attention calls take
  norm_backward    its gradients, the weight's and bias's sums over the rows among them

With `own` false, `run` computes them by elementary torch operations in 32 bits; with `own` true it calls the library.
Values are seeded normals: scores of unit variance, gradients of the size of one value, weights around one.
"""

import math

import torch

own = False

_DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attn(kind, B, H, T, D, **opts):
    c = {"kind": kind, "B": B, "H": H, "T": T, "D": D}
    if kind == "sparse_backward":
        c.update(block=64, pattern="image", frames=1, grid_h=0, grid_w=0, n_text=0, keep=1, per_head=False,
                 ratio=True, rho_delta=0.0)
    c.update(opts)
    return c


def _norm(kind, layout, B, N, H, W, **opts):
    """layout "heads": rows are the H heads of N tokens, read from a packed projection [B, N, 3, H, W] and written
    as [B, H, N, W]; "tokens": rows are the tokens [B, N, W] (H is 1)."""
    c = {"kind": kind, "layout": layout, "B": B, "N": N, "H": H, "W": W, "type": "bf16", "weight": "fp32",
         "per_sample": False, "eps": 1e-6}
    c.update(opts)
    return c


def listed():
    cases = {
        # smallest call: two heads of 256 tokens, launch and host time
        "tiny_full": _attn("full_backward", 1, 2, 256, 64),
        # PixArt-alpha 512 px: a short layer, 72-wide heads
        "pixart_alpha_512_full": _attn("full_backward", 2, 16, 1024, 72),
        # PixArt-Sigma 1024 px: an ordinary image layer
        "pixart_sigma_1024_full": _attn("full_backward", 2, 16, 4096, 72),
        # CogVideoX-2B: a video layer, the largest call
        "cogvideox_2b_full": _attn("full_backward", 2, 30, 17776, 64),
        # fine-tuning through the sparse path at 512 px: 32-token blocks
        "pixart_alpha_512_sparse": _attn("sparse_backward", 2, 16, 1024, 72, block=32, grid_h=32, grid_w=32, keep=1),
        # the longest image layer
        "pixart_sigma_2k_sparse": _attn("sparse_backward", 2, 16, 16384, 72, grid_h=128, grid_w=128, keep=8,
                                        rho_delta=0.02),
        # the video layer: text key blocks are kept by every query block, so key blocks differ widely in work
        "cogvideox_2b_sparse": _attn("sparse_backward", 2, 30, 17776, 64, pattern="video", frames=13, grid_h=30,
                                     grid_w=45, n_text=226, keep=5),
        # a ragged layer with another mask for each head, new in every step, and no reshape
        "ragged_per_head_sparse": _attn("sparse_backward", 1, 12, 5285, 64, pattern="random", keep=9, per_head=True,
                                        ratio=False),
        # queries of the video layer before attention: each head's row, out of the packed projection
        "cogvideox_2b_heads_norm": _norm("norm", "heads", 2, 17776, 30, 64),
        # tokens of a short layer, scaled and shifted for each sample, 16-bit weights
        "pixart_alpha_512_tokens_norm": _norm("norm", "tokens", 2, 1024, 1, 1152, type="fp16", weight="fp16",
                                              per_sample=True),
        # gradients of the video layer's head norm: into the packed projection's gradient
        "cogvideox_2b_heads_norm_backward": _norm("norm_backward", "heads", 2, 17776, 30, 64),
        # gradients of an ordinary layer's token norm, weights for each sample
        "pixart_sigma_1024_tokens_norm_backward": _norm("norm_backward", "tokens", 2, 4096, 1, 1152, per_sample=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


_KINDS = ["full_backward"] * 3 + ["sparse_backward"] * 4 + ["norm"] * 2 + ["norm_backward"] * 3


def draw(rng):
    most = max(_cost(c) for c in listed())

    def spread(lo, hi):
        return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    while True:
        kind = rng.choice(_KINDS)
        B = rng.choice([1, 2, 2, 3])
        if kind == "full_backward":
            c = _attn(kind, B, rng.randint(1, 30), spread(16, 17776), rng.choice([64, 72]))
        elif kind == "sparse_backward":
            block, pattern = rng.choice([32, 64, 64]), rng.choice(["image", "video", "random"])
            frames, n_text = (rng.randint(2, 13), rng.randint(0, 256)) if pattern == "video" else (1, 0)
            area = spread(64, 17776) / frames
            h = max(1, round(math.sqrt(area) * math.exp(rng.uniform(-0.4, 0.4))))
            w = max(1, round(area / h))
            T = n_text + frames * h * w
            n_blk = -(-T // block)
            if T < 64:
                continue
            c = _attn(kind, B, rng.randint(1, 30), T, rng.choice([64, 72]), block=block, pattern=pattern,
                      frames=frames, grid_h=h, grid_w=w, n_text=n_text,
                      keep=max(1, round(n_blk * rng.choice([1 / 32, 1 / 32, 1 / 16, 1 / 8]))),
                      ratio=rng.random() < 0.6, rho_delta=rng.choice([0.0, 0.02]))
            c["per_head"] = pattern == "random" and rng.random() < 0.5
        else:
            layout = rng.choice(["heads", "tokens"])
            H, W = (rng.randint(1, 30), rng.choice([64, 72])) if layout == "heads" else (1, spread(16, 8192))
            if rng.random() < 0.6:
                W = -(-W // 8) * 8
            dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
            c = _norm(kind, layout, B, spread(4, 17776), H, W, type=dtype, weight=rng.choice(["fp32", dtype]),
                      per_sample=layout == "tokens" and rng.random() < 0.4, eps=rng.choice([1e-5, 1e-6]))
        if _cost(c) <= most:
            return c


def _cost(c):
    """Work of one pass in bf16 matrix operations: its own, or its bytes at 300 operations a byte."""
    w = work(c)
    return max(w["flops"], 300.0 * w["bytes"])


def work(c):
    if c["kind"] in ("norm", "norm_backward"):
        rows, W = c["B"] * c["N"] * c["H"], c["W"]
        size = _TYPES[c["type"]].itemsize
        vectors = (c["B"] if c["per_sample"] else 1) * W
        if c["kind"] == "norm":
            return {"bytes": 2 * rows * W * size + 2 * vectors * _TYPES[c["weight"]].itemsize + 8 * rows,
                    "flops": 8 * rows * W}
        return {"bytes": 3 * rows * W * size + vectors * (_TYPES[c["weight"]].itemsize + 8) + 8 * rows,
                "flops": 16 * rows * W}
    heads, T, D = c["B"] * c["H"], c["T"], c["D"]
    sparse = c["kind"] == "sparse_backward"
    pairs = _kept_pairs(c) if sparse else heads * T * T
    stats = 8 + (8 if sparse and c["ratio"] else 0)  # m, l, and rho with its gradient
    return {"bytes": heads * T * (8 * D * 2 + stats), "flops": 10 * pairs * D}


# ---- the block mask -----------------------------------------------------------------------


def _blocks(c):
    """bool [n_masks, n, n]: the key blocks that each query block keeps."""
    T, bs, nt = c["T"], c["block"], c["n_text"]
    n = -(-T // bs)
    if c["pattern"] == "random":  # the diagonal and `keep` - 1 others, drawn
        g = torch.Generator().manual_seed(T + 131 * c["keep"])
        order = torch.rand((c["H"] if c["per_head"] else 1, n, n), generator=g)
        order.diagonal(dim1=1, dim2=2).fill_(2.0)
    else:  # the nearest by the blocks' mean position; text blocks always
        t = torch.arange(n * bs).reshape(n, bs).clamp(max=T - 1) - nt
        hw = c["grid_h"] * c["grid_w"]
        pos = torch.stack([t // hw, (t // c["grid_w"]) % c["grid_h"], t % c["grid_w"]], -1).double().mean(1)
        order = -(pos[:, None] - pos[None]).square().sum(-1)[None] - 1e-9 * torch.arange(n).double()
        order.diagonal(dim1=1, dim2=2).fill_(1.0)
    n_tb = -(-nt // bs)
    order[:, :, :n_tb] = -math.inf
    top = order.topk(min(c["keep"], n), dim=-1).indices
    kept = torch.zeros(order.shape, dtype=torch.bool).scatter_(2, top, True)
    kept[:, :, :n_tb] = True
    kept[:, :n_tb, n_tb:] = False
    return kept


def _kept_pairs(c):
    """Pairs of a query and a key that a call over this mask takes, over all heads."""
    kept = _blocks(c)
    n = kept.shape[1]
    size = torch.full((n,), c["block"])
    size[-1] = c["T"] - (n - 1) * c["block"]
    return int((size[:, None] * size * kept).sum()) * (c["B"] * c["H"] // kept.shape[0])


def _mask(c):
    """The block mask as a program holds it: CSR arrays on the GPU."""
    kept = _blocks(c)
    counts = kept.sum(2)
    row_ptr = torch.zeros((kept.shape[0], kept.shape[1] + 1), dtype=torch.int64)
    row_ptr[:, 1:] = counts.reshape(-1).cumsum(0).reshape(counts.shape)
    row_ptr[1:, 0] = row_ptr[:-1, -1]
    return row_ptr.int().to(_DEV).reshape(-1), kept.nonzero()[:, 2].int().to(_DEV), kept.shape[0], kept.shape[1]


def _handle(m, block):
    import paper_2505_22918_amd as rt

    row_ptr, col_idx, n_masks, n = m
    return rt.BlockMask(row_ptr, col_idx, block, n, col_idx.numel(), n_masks)


# ---- inputs -------------------------------------------------------------------------------


def prepare(c, seed):
    g = torch.Generator(device=_DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=_DEV)

    s = {"case": c}
    if c["kind"] in ("norm", "norm_backward"):
        B, N, H, W, dt, wt = c["B"], c["N"], c["H"], c["W"], _TYPES[c["type"]], _TYPES[c["weight"]]
        packed = (normal(B, N, 3, H, W) if c["layout"] == "heads" else normal(B, N, W)).mul_(1.5).add_(0.3).to(dt)
        heads = c["layout"] == "heads"
        s["x"] = packed[:, :, 0].transpose(1, 2) if heads else packed
        shape = (B, W) if c["per_sample"] else (W,)
        s["weight"], s["bias"] = (1 + 0.2 * normal(*shape)).to(wt), (0.2 * normal(*shape)).to(wt)
        if c["kind"] == "norm_backward":
            x = s["x"].double()
            s["mean"] = x.mean(-1).float()
            s["rstd"] = (x.var(-1, unbiased=False) + c["eps"]).rsqrt().float()
            s["dy"] = normal(*s["x"].shape).to(dt)
            s["dx"] = torch.zeros_like(packed)[:, :, 0].transpose(1, 2) if heads else torch.empty_like(packed)
        return s
    shape = (c["B"], c["H"], c["T"], c["D"])
    s["q"], s["k"], s["v"], s["do"] = (normal(*shape).bfloat16() for _ in range(4))
    if c["kind"] == "full_backward":
        s["o"], s["m"], s["l"] = _full_forward(s["q"], s["k"], s["v"])
        return s
    s["mask"] = _mask(c)
    s["o"], s["m"], s["l"] = _sparse_forward(s["q"], s["k"], s["v"], s["mask"], c["block"])
    if c["ratio"]:  # scattered around the kept share, some close to one
        share = s["mask"][1].numel() / (s["mask"][2] * s["mask"][3] ** 2)
        s["rho"] = (share * torch.exp(0.5 * normal(*shape[:3]))).clamp(max=1.0)
    if own and not c["per_head"]:  # a program with one mask for a run keeps its handle
        s["handle"] = _handle(s["mask"], c["block"])
    return s


# ---- the plain form -----------------------------------------------------------------------


def _heads_at_once(T):
    return max(1, (1 << 31) // (T * T))


def _full_forward(q, k, v):
    B, H, T, D = q.shape
    o, m, l = torch.empty_like(q).reshape(-1, T, D), q.new_empty((B * H, T), dtype=torch.float32), None
    l = torch.empty_like(m)
    n = _heads_at_once(T)
    for i in range(0, B * H, n):
        Q, K, V = (x.reshape(-1, T, D)[i:i + n].float() for x in (q, k, v))
        S = Q @ K.transpose(1, 2) / math.sqrt(D)
        m[i:i + n] = S.amax(-1)
        S.sub_(m[i:i + n, :, None]).exp_()
        l[i:i + n] = S.sum(-1)
        o[i:i + n] = (S @ V / l[i:i + n, :, None]).to(o.dtype)
    return o.reshape(q.shape), m.reshape(B, H, T), l.reshape(B, H, T)


def _full_backward(s):
    B, H, T, D = s["q"].shape
    dq, dk, dv = (torch.empty_like(s["q"]).reshape(-1, T, D) for _ in range(3))
    n = _heads_at_once(T)
    for i in range(0, B * H, n):
        Q, K, V, O, dO = (s[x].reshape(-1, T, D)[i:i + n].float() for x in ("q", "k", "v", "o", "do"))
        m, l = (s[x].reshape(-1, T, 1)[i:i + n] for x in ("m", "l"))
        P = (Q @ K.transpose(1, 2) / math.sqrt(D)).sub_(m).exp_().div_(l)
        dv[i:i + n] = (P.transpose(1, 2) @ dO).to(dv.dtype)
        P *= (dO @ V.transpose(1, 2)).sub_((dO * O).sum(-1, keepdim=True))
        dq[i:i + n] = (P @ K / math.sqrt(D)).to(dq.dtype)
        dk[i:i + n] = (P.transpose(1, 2) @ Q / math.sqrt(D)).to(dk.dtype)
    return {"dq": dq.reshape(s["q"].shape), "dk": dk.reshape(s["q"].shape), "dv": dv.reshape(s["q"].shape)}


def _kept_lists(mask, heads, T, bs):
    """For each head and query block its kept key blocks in a list as long as the longest (their number in all heads'
    key blocks, [BH, n, most]), and which of their keys there are ([BH, n, 1, most * bs])."""
    row_ptr, col_idx, n_masks, n = mask
    row_ptr = row_ptr.reshape(n_masks, n + 1).long()
    counts = row_ptr[:, 1:] - row_ptr[:, :-1]
    most = int(counts.max())
    at = torch.arange(most, device=_DEV)
    there = at < counts[..., None]
    cols = col_idx.long()[(row_ptr[:, :-1, None] + at).clamp(max=col_idx.numel() - 1)]
    keys = there[..., None] & (cols[..., None] * bs + torch.arange(bs, device=_DEV) < T)
    which = torch.arange(heads, device=_DEV) % n_masks
    cols = torch.where(there, cols, 0)[which] + n * torch.arange(heads, device=_DEV)[:, None, None]
    return cols, keys.reshape(n_masks, n, 1, most * bs)[which]


def _in_blocks(x, bs):
    """[B, H, T, ..] as 32-bit blocks [BH * n, bs, ..], zeros past T."""
    T = x.shape[2]
    x = x.float().flatten(0, 1)
    pad = torch.zeros((x.shape[0], -T % bs, *x.shape[2:]), device=_DEV)
    return torch.cat([x, pad], 1).reshape(-1, bs, *x.shape[2:])


def _out_of_blocks(x, like):
    B, H, T, D = like.shape
    return x.reshape(B * H, -1, D)[:, :T].reshape(like.shape)


def _sparse_scores(q, k, mask, bs):
    B, H, T, D = q.shape
    cols, keys = _kept_lists(mask, B * H, T, bs)
    n = cols.shape[1]
    Q = _in_blocks(q, bs).reshape(B * H, n, bs, D)
    K = _in_blocks(k, bs)[cols].reshape(B * H, n, -1, D)
    S = Q @ K.transpose(2, 3) / math.sqrt(D)
    return Q, K, S.masked_fill_(~keys, -math.inf), cols


def _sparse_forward(q, k, v, mask, bs):
    B, H, T, D = q.shape
    _, _, S, cols = _sparse_scores(q, k, mask, bs)
    m = S.amax(-1)
    P = S.sub_(m[..., None]).exp_()
    l = P.sum(-1)
    O = P @ _in_blocks(v, bs)[cols].reshape(B * H, S.shape[1], -1, D) / l[..., None]
    m, l = (x.reshape(B * H, -1)[:, :T].reshape(B, H, T).contiguous() for x in (m, l))
    return _out_of_blocks(O, q).bfloat16(), m, l


def _sparse_backward(s):
    q, bs = s["q"], s["case"]["block"]
    B, H, T, D = q.shape
    Q, K, S, cols = _sparse_scores(q, s["k"], s["mask"], bs)
    n = Q.shape[1]
    blocks = lambda x: _in_blocks(x, bs).reshape(B * H, n, bs, *x.shape[3:])  # noqa: E731
    delta = (s["do"].float() * s["o"].float()).sum(-1)
    w = torch.ones_like(s["m"])
    out = {}
    if "rho" in s:
        ramped = s["rho"] + s["case"]["rho_delta"]
        w = ramped.clamp(max=1.0)
        out["drho"] = torch.where(ramped <= 1.0, delta, 0.0)
    V, dO = _in_blocks(s["v"], bs)[cols].reshape(B * H, n, -1, D), blocks(s["do"])
    factor = blocks(w / s["l"])[..., None]
    P = S.sub_(blocks(s["m"])[..., None]).exp_().mul_(factor)

    def over_queries(x):  # sums of [BH, n, most * bs, D] over the query blocks that keep a key block
        y = torch.zeros((B * H * n, bs * D), device=_DEV)
        return y.index_add_(0, cols.reshape(-1), x.reshape(-1, bs * D))

    out["dv"] = _out_of_blocks(over_queries(P.transpose(2, 3) @ dO), q).bfloat16()
    P *= (dO @ V.transpose(2, 3)).sub_(blocks(delta)[..., None])
    out["dq"] = _out_of_blocks(P @ K / math.sqrt(D), q).bfloat16()
    out["dk"] = _out_of_blocks(over_queries(P.transpose(2, 3) @ Q / math.sqrt(D)), q).bfloat16()
    return out


def _per_row(w, x):
    """A weight of one vector, or one for each sample, against x [B, .., W]."""
    w = w.float()
    return w if w.dim() == 1 else w.reshape(w.shape[0], *[1] * (x.dim() - 2), -1)


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(-1, keepdim=True) + s["case"]["eps"]).rsqrt()
    y = d * rstd * _per_row(s["weight"], x) + _per_row(s["bias"], x)
    return {"y": y.to(s["x"].dtype).contiguous(), "mean": mean[..., 0].contiguous(), "rstd": rstd[..., 0].contiguous()}


def _plain_norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    rstd = s["rstd"][..., None]
    xh = (x - s["mean"][..., None]) * rstd
    g = dy * _per_row(s["weight"], x)
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    rows = list(range(1 if s["weight"].dim() == 2 else 0, x.dim() - 1))
    s["dx"].copy_(dx)
    return {"dx": s["dx"], "dweight": (dy * xh).sum(rows), "dbias": dy.sum(rows)}


# ---- one pass -----------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if own:
        import paper_2505_22918_amd as rt

        if c["kind"] == "full_backward":
            return dict(zip(("dq", "dk", "dv"), rt.attn_full_backward(s["q"], s["k"], s["v"], s["o"], s["m"], s["l"],
                                                                      s["do"])))
        if c["kind"] == "sparse_backward":
            # a mask of its own for each head is new in each step: its handle is part of the pass
            mask = s["handle"] if "handle" in s else _handle(s["mask"], c["block"])
            out = rt.attn_sparse_backward(s["q"], s["k"], s["v"], s["o"], s["m"], s["l"], s["do"], mask,
                                          rho=s.get("rho"), rho_delta=c["rho_delta"])
            return dict(zip(("dq", "dk", "dv", "drho"), out))
        if c["kind"] == "norm":
            return dict(zip(("y", "mean", "rstd"), rt.layer_norm(s["x"], s["weight"], s["bias"], eps=c["eps"],
                                                                 stats=True)))
        return dict(zip(("dx", "dweight", "dbias"), rt.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"],
                                                                           s["weight"], out=s["dx"])))
    if c["kind"] == "full_backward":
        return _full_backward(s)
    if c["kind"] == "sparse_backward":
        return _sparse_backward(s)
    return _plain_norm(s) if c["kind"] == "norm" else _plain_norm_backward(s)


# ---- in 64 bits ---------------------------------------------------------------------------


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] in ("norm", "norm_backward"):
        return _exact_norm(c, s)
    B, H, T, D = s["q"].shape
    ratio = c["kind"] == "sparse_backward" and c["ratio"]
    names = ("dq", "dk", "dv") + (("drho",) if ratio else ())
    out = {x: [] for x in names}
    for h in range(B * H):
        q, k, v, o, do = (s[x].flatten(0, 1)[h].double() for x in ("q", "k", "v", "o", "do"))
        m, l = (s[x].flatten(0, 1)[h].double() for x in ("m", "l"))
        A = torch.exp(torch.mm(q, k.t()) * D ** -0.5 - m[:, None]) / l[:, None]
        if c["kind"] == "sparse_backward":
            row_ptr, col_idx, n_masks, n = s["mask"]
            first = row_ptr.reshape(n_masks, n + 1)[h % n_masks]
            kept = torch.zeros((n, n), dtype=torch.bool, device=_DEV)
            rows = torch.repeat_interleave(torch.arange(n, device=_DEV), (first[1:] - first[:-1]).long())
            kept[rows, col_idx[int(first[0]):int(first[-1])].long()] = True
            tokens = torch.arange(T, device=_DEV) // c["block"]
            A = A * kept[tokens][:, tokens]
        inner = torch.einsum("td,td->t", do, o)
        gain = torch.ones_like(inner)
        if ratio:
            # the ramped ratio is a 32-bit sum of its two 32-bit terms
            ramped = (s["rho"].flatten(0, 1)[h] + c["rho_delta"]).double()
            gain = torch.minimum(ramped, gain)
            out["drho"].append(inner * (ramped <= 1))
        A = A * gain[:, None]
        out["dv"].append(torch.mm(A.t(), do).cpu())
        A = A * (torch.mm(do, v.t()) - inner[:, None])
        out["dq"].append((torch.mm(A, k) * D ** -0.5).cpu())
        out["dk"].append((torch.mm(A.t(), q) * D ** -0.5).cpu())
    return {x: torch.stack(y).reshape(s["m"].shape if x == "drho" else s["q"].shape) for x, y in out.items()}


def _exact_norm(c, s):
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    if c["per_sample"]:
        w, b = w[:, None], b[:, None]
    W = c["W"]
    if c["kind"] == "norm":
        mean = x.sum(-1) / W
        rstd = ((x - mean[..., None]).pow(2).sum(-1) / W + c["eps"]) ** -0.5
        return {"y": ((x - mean[..., None]) * rstd[..., None] * w + b), "mean": mean, "rstd": rstd}
    dy, mean, rstd = s["dy"].double(), s["mean"].double()[..., None], s["rstd"].double()[..., None]
    xh = (x - mean) * rstd
    first = (dy * w).sum(-1, keepdim=True)
    second = (dy * w * xh).sum(-1, keepdim=True)
    over = tuple(range(1 if c["per_sample"] else 0, x.dim() - 1))
    return {"dx": rstd * (dy * w - (first + xh * second) / W), "dweight": (dy * xh).sum(over), "dbias": dy.sum(over)}
