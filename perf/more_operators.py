"""Rotary positions and differential attention, as they are measured: what follows the norm of queries and keys.

  rope             rotation of heads' rows by the angles of their positions
  rope_backward    its gradient: the inverse rotation
  diff             differential attention, the difference of two softmax maps with a learned weight
  diff_backward    its gradients for queries, keys, values and the weight

With `own` false, `run` computes them by elementary torch operations in 32 bits (angles in 64); with `own` true it calls
the library.  Values are seeded normals: scores of unit variance, gradients of the size of one value.
"""

import math

import torch

own = False

_DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _rope(kind, B, H, T, D, **opts):
    """H heads of T tokens, `rot` of their D elements rotated.  packed: queries and keys of a packed projection
    [B, T, 3, H, D], both in one call (2 H heads).  axes 3: a grid of frames, rows and columns behind n_text text
    tokens at position 0, the elements split over the axes; else one axis from position `start` on, for each sample from
    another one where per_sample."""
    c = {"kind": kind, "B": B, "H": H, "T": T, "D": D, "rot": D, "layout": "interleaved", "type": "bf16",
         "packed": False, "axes": 1, "frames": 1, "grid_h": 1, "grid_w": 1, "n_text": 0, "start": 0, "per_sample": False,
         "base": 10000.0, "scaling": "none", "factor": 1.0}
    c.update(opts)
    return c


def _diff(kind, B, H, Tq, Tk, D, **opts):
    """H heads: 2 H maps of D wide queries and keys, values 2 D wide.  lens "ragged": each sample has a number of keys
    of its own, the last of four and more none.  per_head: a weight for each head, else one for all.  stats: the forward
    call also returns what its gradient needs."""
    c = {"kind": kind, "B": B, "H": H, "Tq": Tq, "Tk": Tk, "D": D, "lens": "all", "per_head": True, "stats": True}
    c.update(opts)
    return c


def listed():
    cases = {
        # smallest call: a token of each of four sequences, launch and host time
        "token_rope": _rope("rope", 4, 16, 1, 72, layout="half", start=4095, per_sample=True),
        # CogVideoX-2B: queries and keys of the video layer, out of the packed projection
        "cogvideox_2b_rope": _rope("rope", 2, 30, 17776, 64, packed=True, axes=3, frames=13, grid_h=30, grid_w=45,
                                   n_text=226),
        # a long context far from its start, in 32 bits: positions scaled by frequency bands
        "far_rope": _rope("rope", 1, 30, 8191, 64, layout="half", type="fp32", start=1000003, base=500000.0,
                          scaling="yarn", factor=16.0),
        # gradient of the longest image layer, two thirds of each head rotated
        "pixart_sigma_2k_rope_backward": _rope("rope_backward", 2, 16, 16384, 72, rot=48, layout="half", type="fp16",
                                               scaling="linear", factor=4.0),
        # smallest layer
        "tiny_diff": _diff("diff", 1, 1, 256, 256, 64),
        # one new token a sequence over the keys of a long one so far, of another length for each
        "token_diff": _diff("diff", 8, 15, 1, 8192, 64, lens="ragged", stats=False),
        # image tokens over a padded batch of text tokens, one weight for the layer
        "text_diff": _diff("diff", 4, 8, 4096, 226, 72, lens="ragged", per_head=False),
        # the video layer, the largest call
        "cogvideox_2b_diff": _diff("diff", 2, 15, 17776, 17776, 64),
        # gradients of a short layer
        "pixart_alpha_512_diff_backward": _diff("diff_backward", 2, 8, 1024, 1024, 72),
        # gradients of an ordinary image layer
        "pixart_sigma_1024_diff_backward": _diff("diff_backward", 2, 8, 4096, 4096, 72),
        # odd sizes, padded keys, one weight for the layer
        "ragged_diff_backward": _diff("diff_backward", 5, 3, 2734, 1175, 64, lens="ragged", per_head=False),
        # gradients of the video layer
        "cogvideox_2b_diff_backward": _diff("diff_backward", 2, 15, 17776, 17776, 64),
    }
    return [dict(c, name=n) for n, c in cases.items()]


_KINDS = ["rope"] * 2 + ["rope_backward"] + ["diff"] * 3 + ["diff_backward"] * 3


def draw(rng):
    most = max(_cost(c) for c in listed())

    def spread(lo, hi):
        return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    while True:
        kind = rng.choice(_KINDS)
        B = rng.choice([1, 2, 2, 3, 5, 8])
        if kind in ("rope", "rope_backward"):
            D = rng.choice([64, 72, 128, 2 * rng.randint(4, 96)])
            c = _rope(kind, B, rng.randint(1, 30), spread(1, 17776), D, layout=rng.choice(["interleaved", "half"]),
                      type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), packed=rng.random() < 0.5,
                      start=rng.choice([0, 0, spread(1, 2000000)]), per_sample=rng.random() < 0.3,
                      base=rng.choice([10000.0, 500000.0]), scaling=rng.choice(["none", "linear", "ntk", "yarn"]),
                      factor=rng.choice([2.0, 4.0, 16.0]))
            if rng.random() < 0.3:
                c["rot"] = 2 * rng.randint(2, D // 2)
            if rng.random() < 0.4 and c["rot"] >= 12:
                frames, area = rng.randint(1, 13), c["T"]
                h = max(1, round(math.sqrt(area / frames)))
                w = max(1, round(area / frames / h))
                n_text = rng.randint(0, 226)
                c.update(axes=3, frames=frames, grid_h=h, grid_w=w, n_text=n_text, T=n_text + frames * h * w, start=0,
                         per_sample=False)
        else:
            Tq = spread(1, 17776)
            Tk = Tq if rng.random() < 0.5 else spread(1, 17776)
            if kind == "diff" and rng.random() < 0.25:
                Tq = 1
            c = _diff(kind, B, rng.randint(1, 15), Tq, Tk, rng.choice([64, 72]), lens=rng.choice(["all", "ragged"]),
                      per_head=rng.random() < 0.7, stats=kind == "diff_backward" or rng.random() < 0.5)
        if _cost(c) <= most:
            return c


def _cost(c):
    """Work of one pass in bf16 matrix operations: its own, or its bytes at 300 operations a byte."""
    w = work(c)
    return max(w["flops"], 300.0 * w["bytes"])


def work(c):
    if c["kind"] in ("rope", "rope_backward"):
        rows = c["B"] * c["H"] * (2 if c["packed"] else 1) * c["T"]
        positions = (c["B"] if c["per_sample"] else 1) * c["T"] * c["axes"] * 8
        return {"bytes": 2 * rows * c["D"] * _TYPES[c["type"]].itemsize + positions, "flops": 3 * rows * c["rot"]}
    B, H, Tq, Tk, D = c["B"], c["H"], c["Tq"], c["Tk"], c["D"]
    keys = sum(_key_counts(c))
    q, kv, o = B * H * Tq * 2 * D * 2, H * keys * 4 * D * 2, B * H * Tq * 2 * D * 2
    stats = B * 2 * H * Tq * 8
    pairs = H * Tq * keys
    if c["kind"] == "diff":
        more = o + stats if c["stats"] else 0
        return {"bytes": q + kv + o + more, "flops": pairs * D * (12 if c["stats"] else 8)}
    return {"bytes": 2 * q + kv + B * H * Tk * 4 * D * 2 + 3 * o + stats, "flops": 20 * pairs * D}


def _key_counts(c):
    """The number of keys of each sample."""
    if c["lens"] == "all":
        return [c["Tk"]] * c["B"]
    g = torch.Generator().manual_seed(c["Tk"] + 131 * c["B"])
    n = [c["Tk"]] + torch.randint(1, c["Tk"] + 1, (c["B"] - 1,), generator=g).tolist()
    if c["B"] > 3:
        n[-1] = 0
    return n


def _axis_widths(c):
    if c["axes"] == 1:
        return [c["rot"]]
    first = 2 * (c["rot"] // 8)
    second = 2 * ((c["rot"] - first) // 4)
    return [first, second, c["rot"] - first - second]


_ORIGINAL = 8192  # positions that the unscaled frequencies were made for


def _frequencies(c):
    """Radians a position of every pair and the axis of each (on the host), and the factor of cosines and sines."""
    freq, axis, s = [], [], c["factor"]
    for a, w in enumerate(_axis_widths(c)):
        base = c["base"]
        if c["scaling"] == "ntk" and w > 2:
            base = base * s ** (w / (w - 2))
        f = torch.tensor(base, dtype=torch.float64) ** (-torch.arange(0, w, 2, dtype=torch.float64) / w)
        if c["scaling"] == "linear":
            f = f / s
        if c["scaling"] == "yarn":
            g = ((_ORIGINAL * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
            f = g * f + (1 - g) * f / s
        freq.append(f)
        axis += [a] * (w // 2)
    return torch.cat(freq), torch.tensor(axis), 0.1 * math.log(s) + 1 if c["scaling"] == "yarn" else 1.0


def _positions(c):
    """int64 [T], or [B, T] per sample, or [T, 3] of a grid."""
    if c["axes"] == 1:
        p = torch.arange(c["T"]) + c["start"]
        return torch.stack([p + 977 * b for b in range(c["B"])]) if c["per_sample"] else p
    t = torch.arange(c["T"] - c["n_text"])
    hw = c["grid_h"] * c["grid_w"]
    grid = torch.stack([t // hw, t // c["grid_w"] % c["grid_h"], t % c["grid_w"]], -1)
    return torch.cat([torch.zeros((c["n_text"], 3), dtype=torch.int64), grid])


# ---- inputs -------------------------------------------------------------------------------


def prepare(c, seed):
    g = torch.Generator(device=_DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=_DEV)

    s = {"case": c}
    if c["kind"] in ("rope", "rope_backward"):
        B, H, T, D, dt = c["B"], c["H"], c["T"], c["D"], _TYPES[c["type"]]
        if c["packed"]:
            s["x"] = normal(B, T, 3, H, D).to(dt)[:, :, :2].flatten(2, 3).transpose(1, 2)
            if c["kind"] == "rope_backward":  # into the packed projection's gradient
                s["dx"] = torch.zeros((B, T, 3, H, D), dtype=dt, device=_DEV)[:, :, :2].flatten(2, 3).transpose(1, 2)
        else:
            s["x"] = normal(B, H, T, D).to(dt)
        if c["kind"] == "rope_backward":  # a gradient comes as attention's gradients are laid out
            s["x"] = s["x"].contiguous()
        s["positions"] = _positions(c).to(_DEV)
        freq, axis, s["amplitude"] = _frequencies(c)
        s["freq"], s["axis"] = freq.to(_DEV), axis.to(_DEV)
        if own:
            import paper_2505_22918_amd as rt

            s["plan"] = rt.rope_plan(c["rot"], base=c["base"], widths=_axis_widths(c), layout=c["layout"],
                                     scaling=None if c["scaling"] == "none" else c["scaling"], factor=c["factor"],
                                     original=_ORIGINAL)
        return s
    B, H, Tq, Tk, D = c["B"], c["H"], c["Tq"], c["Tk"], c["D"]
    s["q"], s["k"] = normal(B, 2 * H, Tq, D).bfloat16(), normal(B, 2 * H, Tk, D).bfloat16()
    s["v"] = normal(B, H, Tk, 2 * D).bfloat16()
    s["lam"] = 0.5 + 0.15 * normal(H if c["per_head"] else 1)
    s["k_lens"] = None if c["lens"] == "all" else torch.tensor(_key_counts(c), dtype=torch.int32, device=_DEV)
    if c["kind"] == "diff_backward":
        s["do"] = normal(B, H, Tq, 2 * D).bfloat16()
        s.update(_plain_diff(s))
    return s


# ---- the plain form -----------------------------------------------------------------------


def _plain_rope(s, sign):
    c, x = s["case"], s["x"].float()
    P = c["rot"] // 2
    p = s["positions"].double()
    p = p[..., None] if c["axes"] == 1 else p
    angle = p[..., s["axis"]] * s["freq"]
    if c["per_sample"]:
        angle = angle[:, None]
    cos, sin = (s["amplitude"] * f(angle) for f in (torch.cos, torch.sin))
    cos, sin = cos.float(), (sign * sin).float()
    y = x.clone(memory_format=torch.contiguous_format)
    one, two = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if c["layout"] == "interleaved" else (slice(0, P), slice(P, 2 * P))
    a, b = x[..., one], x[..., two]
    y[..., one] = a * cos - b * sin
    y[..., two] = a * sin + b * cos
    if "dx" in s:
        return s["dx"].copy_(y)
    return y.to(s["x"].dtype)


def _heads_at_once(Tq, Tk):
    return max(1, (1 << 30) // (Tq * Tk))


def _probabilities(s, b, i, n, m=None, l=None):
    """exp(scores - m) of sample b, heads i .. i + n - 1, [n, 2, Tq, Tk] with m and l, or over l where these are given."""
    Q, K = (s[x][b].float().unflatten(0, (-1, 2))[i:i + n] for x in ("q", "k"))
    S = (Q @ K.transpose(2, 3)).div_(math.sqrt(s["q"].shape[-1]))
    if s["k_lens"] is not None:
        S.masked_fill_(torch.arange(S.shape[-1], device=_DEV) >= s["k_lens"][b], -math.inf)
    if m is None:
        m = S.amax(-1)
        S.sub_(torch.where(m == -math.inf, 0.0, m)[..., None]).exp_()
        return S, m, S.sum(-1)
    S.sub_(torch.where(m == -math.inf, 0.0, m)[..., None]).exp_()
    return S.mul_(torch.where(l > 0, 1 / l, 0.0)[..., None])


def _weights(s):
    H = s["v"].shape[1]
    return s["lam"].expand(H).reshape(H, 1, 1)


def _plain_diff(s):
    c = s["case"]
    B, H, Tq, D2 = c["B"], c["H"], c["Tq"], 2 * c["D"]
    o, o2 = (torch.empty((B, H, Tq, D2), dtype=torch.bfloat16, device=_DEV) for _ in range(2))
    m, l = (torch.empty((B, 2 * H, Tq), device=_DEV) for _ in range(2))
    n = _heads_at_once(Tq, 2 * c["Tk"])
    for b in range(B):
        for i in range(0, H, n):
            P, mi, li = _probabilities(s, b, i, n)
            O = P @ s["v"][b, i:i + n].float()[:, None]
            O *= torch.where(li > 0, 1 / li, 0.0)[..., None]
            o[b, i:i + n] = (O[:, 0] - _weights(s)[i:i + n] * O[:, 1]).bfloat16()
            o2[b, i:i + n] = O[:, 1].bfloat16()
            m[b, 2 * i:2 * (i + n)], l[b, 2 * i:2 * (i + n)] = mi.flatten(0, 1), li.flatten(0, 1)
    return {"o": o, "o2": o2, "m": m, "l": l} if c["stats"] else {"o": o}


def _plain_diff_backward(s):
    c = s["case"]
    dq, dk, dv = (torch.empty_like(s[x]) for x in ("q", "k", "v"))
    B, H, Tq = c["B"], c["H"], c["Tq"]
    scale = 1 / math.sqrt(c["D"])
    delta2 = (s["do"].float() * s["o2"].float()).sum(-1)
    delta1 = (s["do"].float() * s["o"].float()).sum(-1) + _weights(s)[:, 0] * delta2
    m, l = (s[x].unflatten(1, (H, 2)) for x in ("m", "l"))
    n = _heads_at_once(Tq, 2 * c["Tk"])
    for b in range(B):
        for i in range(0, H, n):
            w = _weights(s)[i:i + n]
            P = _probabilities(s, b, i, n, m[b, i:i + n], l[b, i:i + n])
            dO, V = s["do"][b, i:i + n].float(), s["v"][b, i:i + n].float()
            dv[b, i:i + n] = ((P[:, 0] - w * P[:, 1]).transpose(1, 2) @ dO).bfloat16()
            dA = dO @ V.transpose(1, 2)
            P[:, 0] *= dA - delta1[b, i:i + n, :, None]
            P[:, 1] *= (dA - delta2[b, i:i + n, :, None]) * -w
            Q, K = (s[x][b].float().unflatten(0, (-1, 2))[i:i + n] for x in ("q", "k"))
            dq[b, 2 * i:2 * (i + n)] = (P @ K * scale).bfloat16().flatten(0, 1)
            dk[b, 2 * i:2 * (i + n)] = (P.transpose(2, 3) @ Q * scale).bfloat16().flatten(0, 1)
    dlam = -delta2.double().sum((0, 2))
    return {"dq": dq, "dk": dk, "dv": dv, "dlam": (dlam if c["per_head"] else dlam.sum(0, keepdim=True)).float()}


# ---- one pass -----------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if own:
        import paper_2505_22918_amd as rt

        if c["kind"] == "rope":
            return {"y": rt.rope(s["x"], s["positions"], s["plan"])}
        if c["kind"] == "rope_backward":
            return {"dx": rt.rope_backward(s["x"], s["positions"], s["plan"], out=s.get("dx"))}
        if c["kind"] == "diff":
            out = rt.attn_diff(s["q"], s["k"], s["v"], s["lam"], k_lens=s["k_lens"], stats=c["stats"])
            return dict(zip(("o", "o2", "m", "l"), out)) if c["stats"] else {"o": out}
        return dict(zip(("dq", "dk", "dv", "dlam"),
                        rt.attn_diff_backward(s["q"], s["k"], s["v"], s["o"], s["o2"], s["m"], s["l"], s["do"], s["lam"],
                                              k_lens=s["k_lens"])))
    if c["kind"] == "rope":
        return {"y": _plain_rope(s, 1.0)}
    if c["kind"] == "rope_backward":
        return {"dx": _plain_rope(s, -1.0)}
    return _plain_diff(s) if c["kind"] == "diff" else _plain_diff_backward(s)


# ---- in 64 bits ---------------------------------------------------------------------------


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] in ("rope", "rope_backward"):
        return _exact_rope(c, s)
    B, H, D = c["B"], c["H"], c["D"]
    lam = s["lam"].double().expand(H)
    out = {}

    def put(name, value):
        out.setdefault(name, []).append(value.cpu())

    dlam = torch.zeros(H, dtype=torch.float64, device=_DEV)
    for b, keys in enumerate(_key_counts(c)):
        for h in range(H):
            v = s["v"][b, h, :keys].double()
            maps = []
            for i in (2 * h, 2 * h + 1):
                q, k = s["q"][b, i].double(), s["k"][b, i, :keys].double()
                maps.append((q, k, torch.mm(q, k.t()) * D ** -0.5))
            if c["kind"] == "diff":
                parts = []
                for _, _, z in maps:
                    top = z.max(1).values if keys else z.new_full((c["Tq"],), -math.inf)
                    e = torch.exp(z - top[:, None])
                    total = e.sum(1)
                    parts.append(torch.mm(e, v) / total.clamp(min=1e-300)[:, None])
                    if c["stats"]:
                        put("m", top)
                        put("l", total)
                put("o", parts[0] - lam[h] * parts[1])
                if c["stats"]:
                    put("o2", parts[1])
                continue
            do = s["do"][b, h].double()
            inner2 = torch.einsum("td,td->t", do, s["o2"][b, h].double())
            inner1 = torch.einsum("td,td->t", do, s["o"][b, h].double()) + lam[h] * inner2
            dlam[h] -= inner2.sum()
            A = [torch.exp(z - s["m"][b, 2 * h + i].double()[:, None]) / s["l"][b, 2 * h + i].double()[:, None]
                 for i, (_, _, z) in enumerate(maps)]
            rest = c["Tk"] - keys

            def tall(x):  # zeros for the rows past the keys
                return torch.cat([x, x.new_zeros((rest, x.shape[1]))])

            put("dv", tall(torch.mm(A[0].t(), do) - lam[h] * torch.mm(A[1].t(), do)))
            pull = torch.mm(do, v.t())
            for a, (q, k, _), inner, gain in zip(A, maps, (inner1, inner2), (1.0, -lam[h])):
                e = a * (pull - inner[:, None]) * gain
                put("dq", torch.mm(e, k) * D ** -0.5)
                put("dk", tall(torch.mm(e.t(), q) * D ** -0.5))
    like = {"m": s["q"].shape[:3], "l": s["q"].shape[:3], "o": (B, H, c["Tq"], 2 * D), "o2": (B, H, c["Tq"], 2 * D),
            "dq": s["q"].shape, "dk": s["k"].shape, "dv": s["v"].shape}
    out = {x: torch.stack(y).reshape(like[x]) for x, y in out.items()}
    if c["kind"] == "diff_backward":
        out["dlam"] = dlam if c["per_head"] else dlam.sum().reshape(1)
    return out


def _exact_rope(c, s):
    freq, axis, gain = _frequencies(c)
    p = _positions(c).double()
    if c["axes"] == 1:
        p = p.unsqueeze(-1)
    turn = torch.polar(torch.full((), gain, dtype=torch.float64), p[..., axis] * freq).to(_DEV)
    if c["kind"] == "rope_backward":
        turn = turn.conj()
    if c["per_sample"]:
        turn = turn.unsqueeze(1)
    x, rot = s["x"].double(), c["rot"]
    head, tail = x[..., :rot], x[..., rot:]
    if c["layout"] == "half":
        z = turn * torch.complex(*head.chunk(2, dim=-1))
        head = torch.cat([z.real, z.imag], dim=-1)
    else:
        z = turn * torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous())
        head = torch.view_as_real(z).flatten(-2)
    return {"y" if c["kind"] == "rope" else "dx": torch.cat([head, tail], dim=-1)}
