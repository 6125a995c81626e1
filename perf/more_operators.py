"""Timed cases of per-head norms with rotary positions, and of a cache in 4 bits.

Norms and rotation: a projection gives q, k and v of every token, [B, S, H + 2 Hkv, d]. Each head of q and
k is normed over its d values (root mean square, or mean and variance), pairs of its values are turned by
angles position * frequency with positions of one axis or of three (time, height, width), and everything is
laid out as [B, H, S, d]. The cache holds keys and values in e2m1, 128 tokens a page, with a power of two for
every 32 values of a token.

A case is a dict of plain values:
  name    (listed cases only)
  op      "rope"  norms and rotation       "rope_grad"  gradients of the projection and of the norms' weights
          "write" N new tokens of every sequence into the pages, and the values that the cache then holds
          "read"  N tokens from `first` on "attn"       attention of the last N tokens over the cache
  B, H, Hkv, d     batch, query heads, key heads, head dim
  S, norm, layout, axes   rope: tokens; "rms", "layer" or ""; which values are pairs; values of each axis ("32,32,32")
  text, h, w, ragged, far tokens without a position before the video, its grid, lengths that differ, single tokens far along
  N, lo, hi, first cache: tokens of the call, shortest and longest sequence (write: before the call)

Sizes: 720p video (3600 tokens a latent frame; 8 and 24 frames), the CogVideoX-5B head size, and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 128
GROUP = 32  # values of a token that share a scale
EPS = 1e-6


def _rope(op, B, S, H, Hkv, d, norm, layout, axes, text=0, h=1, w=1, ragged=False, far=False, name=None):
    c = {"op": op, "B": B, "S": S, "H": H, "Hkv": Hkv, "d": d, "norm": norm, "layout": layout, "axes": axes,
         "text": text, "h": h, "w": w, "ragged": ragged, "far": far}
    return c if name is None else {"name": name, **c}


def _paged(op, B, H, Hkv, d, N, lo, hi, first=0, name=None):
    c = {"op": op, "B": B, "H": H, "Hkv": Hkv, "d": d, "N": N, "lo": lo, "hi": hi, "first": first}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # One token of 32 sequences, far along: a decoding step's latency.
        _rope("rope", 32, 1, 32, 8, 128, "rms", "halves", "128", far=True, name="rope-token"),
        # A padded batch of short clips with grouped heads, odd length.
        _rope("rope", 2, 777, 6, 2, 64, "layer", "interleaved", "16,24,24", h=9, w=13, ragged=True, name="rope-odd"),
        # A 93-frame 720p layer, all heads.
        _rope("rope", 1, 86400, 24, 24, 96, "rms", "halves", "32,32,32", h=45, w=80, name="rope-93f"),
        # Gradients at the CogVideoX-5B head size: text and one frame and a half.
        _rope("rope_grad", 1, 2251, 12, 12, 64, "layer", "interleaved", "16,24,24", text=226, h=30, w=45,
              name="grad-odd"),
        # Gradients of a 29-frame 720p layer, all heads.
        _rope("rope_grad", 1, 28800, 24, 24, 96, "rms", "halves", "32,32,32", h=45, w=80, name="grad-29f"),
        # One new token of 32 sequences into their pages: latency.
        _paged("write", 32, 8, 8, 128, 1, 200, 30000, name="write4-token"),
        # Three prompts written at once behind what is there.
        _paged("write", 3, 8, 8, 96, 8191, 0, 100, name="write4-prompt"),
        # Some tokens from the middle of short sequences: latency.
        _paged("read", 4, 2, 2, 64, 333, 100, 500, first=77, name="read4-short"),
        # A prefix for the attention of a prompt behind it.
        _paged("read", 2, 8, 8, 128, 30001, 20000, 30001, name="read4-prefix"),
        # A draft of four tokens over short sequences: latency.
        _paged("attn", 3, 12, 4, 64, 4, 700, 1500, name="attn4-draft"),
        # A decoding step of 24 sequences of a thousand to a hundred thousand tokens.
        _paged("attn", 24, 32, 8, 128, 1, 1000, 100000, name="attn4-long"),
        # Eight drafted tokens of each sequence, more rows than one pass over the cache takes.
        _paged("attn", 4, 48, 4, 96, 8, 5000, 20000, name="attn4-rows"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: every operator, head dim, group size, norm, pairing and number of
    axes, one token to long sequences, odd lengths, padded batches."""
    while True:
        op = rng.choice(["rope", "rope", "rope_grad", "rope_grad", "write", "read", "attn", "attn"])
        d = rng.choice([64, 96, 128])
        Hkv = rng.choice([1, 2, 3, 4, 6, 8])
        H = Hkv * rng.choice([1, 1, 2, 3, 4, 8])
        if op in ("rope", "rope_grad"):
            single = op == "rope" and rng.random() < 0.3
            B = _log_int(rng, 1, 64) if single else rng.choice([1, 1, 2, 3, 4])
            S = 1 if single else _log_int(rng, 1, 60000)
            three = not single and rng.random() < 0.6
            if three:
                a, b = 2 * rng.randint(4, d // 8), 2 * rng.randint(4, d // 6)
                axes = "%d,%d,%d" % (a, b, b)
            else:
                axes = str(rng.choice([d, d, d // 2, 2 * rng.randint(4, d // 2)]))
            case = _rope(op, B, S, H, Hkv, d, rng.choice(["rms", "rms", "layer", ""]),
                         rng.choice(["interleaved", "halves", "split"]), axes,
                         text=rng.choice([0, 226]) if three else 0, h=rng.randint(5, 50) if three else 1,
                         w=rng.randint(5, 80) if three else 1, ragged=not single and rng.random() < 0.4, far=single)
        else:
            B = _log_int(rng, 1, 48)
            if op == "attn":
                N = rng.choice([1, 1, 1, 2, 5, 9])
                hi = _log_int(rng, N, 80000)
                lo = rng.randint(min(N, hi), hi)
            else:
                N = _log_int(rng, 1, 6000) if rng.random() < 0.6 else rng.choice([1, 1, 2, 5])
                hi = _log_int(rng, 1, 20000)
                lo = rng.randint(0, hi)
            first = rng.randint(0, hi) if op == "read" and rng.random() < 0.5 else 0
            case = _paged(op, B, H if op == "attn" else Hkv, Hkv, d, N, lo, hi, first)
        w = work(case)
        if w["flops"] <= 5e10 and w["bytes"] <= 8e8 and _elements(case) <= 2e9:
            return case


def _elements(case):
    """Numbers that the plain form holds at once in its largest tensor."""
    B, H, Hkv, d = (case[k] for k in ("B", "H", "Hkv", "d"))
    if case["op"] in ("rope", "rope_grad"):
        return B * case["S"] * (H + 2 * Hkv) * d
    if case["op"] in ("write", "read"):
        return B * Hkv * d * (case["hi"] + 2 * case["N"])
    return B * max(Hkv * d, H * case["N"]) * case["hi"]


def _lens(case):
    """Tokens of each sequence. Cache: from hi down to lo, evenly over the logarithm. Norms: all of them, or
    with ragged from all down to half."""
    B = case["B"]
    if case["op"] in ("rope", "rope_grad"):
        S = case["S"]
        return [S - (b * S) // (2 * B) if case["ragged"] else S for b in range(B)]
    lo, hi = case["lo"], case["hi"]
    f = [(math.log(lo + 1) * b + math.log(hi + 1) * (B - 1 - b)) / max(1, B - 1) for b in range(B)]
    return [min(hi, max(lo, round(math.exp(x)) - 1)) for x in f]


def work(case):
    """What the operator cannot do without: every input read once and every output written once, two
    products of 2 d operations per query-key pair of attention, some operations a value elsewhere."""
    B, H, Hkv, d, op = (case[k] for k in ("B", "H", "Hkv", "d", "op"))
    if op in ("rope", "rope_grad"):
        rows = sum(_lens(case))
        n = rows * (H + 2 * Hkv) * d
        every = B * case["S"] * (H + 2 * Hkv) * d
        if op == "rope":
            return {"bytes": 2.0 * n + 2 * every, "flops": 10.0 * n}
        return {"bytes": 4.0 * n + 2 * every, "flops": 25.0 * n}
    lens, held = _lens(case), d / 2 + d / GROUP  # bytes of a token's keys, or values, of a head
    if op == "write":
        n = 2.0 * B * case["N"] * Hkv
        return {"bytes": n * (4 * d + held), "flops": 6.0 * n * d}
    if op == "read":
        n = 2.0 * sum(max(0, min(case["N"], x - case["first"])) for x in lens) * Hkv
        return {"bytes": n * held + 4.0 * B * case["N"] * Hkv * d, "flops": n * d}
    tokens, rows = sum(lens), B * H * case["N"]
    return {"bytes": 2.0 * tokens * Hkv * held + rows * (4 * d + 4), "flops": 4.0 * d * H * case["N"] * tokens}


# ---------------------------------------------------------------------------------------------
# inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 57)


def _dims(case):
    return tuple(int(x) for x in case["axes"].split(","))


def _inputs(case, seed):
    gen = _gen(seed)
    if case["op"] not in ("rope", "rope_grad"):
        return _pages(case, gen)
    B, S, H, Hkv, d = (case[k] for k in ("B", "S", "H", "Hkv", "d"))
    dims = _dims(case)
    dev = dict(device="cuda")
    x = torch.randn((B, S, H + 2 * Hkv, d), generator=gen, **dev)
    x *= 0.5 + torch.rand((H + 2 * Hkv, d), generator=gen, **dev)  # channels of their own magnitude
    st = {"x": (x + 0.2).to(torch.bfloat16)}
    for name in ("q_weight", "k_weight"):
        st[name] = 1 + 0.2 * torch.randn(d, generator=gen, **dev) if case["norm"] else None
    for name in ("q_bias", "k_bias"):
        st[name] = 0.1 * torch.randn(d, generator=gen, **dev) if case["norm"] == "layer" else None
    if len(dims) == 3:
        t = (torch.arange(S, **dev) - case["text"]).clamp(min=0)
        h, w = case["h"], case["w"]
        at = torch.stack([t // (h * w), t // w % h, t % w], -1)
    elif case["far"]:
        at = torch.randint(0, 1 << 20, (B, S, 1), generator=gen, **dev)
    else:
        at = torch.arange(S, **dev)[:, None]
    st["positions"] = at.to(torch.int32).contiguous()
    st["freqs"] = torch.cat([10000.0 ** (-torch.arange(0, n, 2, dtype=torch.float64, **dev) / n) for n in dims])
    st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, **dev) if case["ragged"] else None
    if case["op"] == "rope_grad":
        for name, heads in (("dq", H), ("dk", Hkv), ("dv", Hkv)):
            st[name] = torch.randn((B, heads, S, d), generator=gen, **dev).to(torch.bfloat16)
    return st


def _pages(case, gen):
    """A cache whose sequences hold their tokens, pages in random places, and the new tokens (write) or the
    queries (attn). Magnitudes differ from channel group to channel group."""
    B, H, Hkv, d, N, op = (case[k] for k in ("B", "H", "Hkv", "d", "N", "op"))
    lens = _lens(case)
    need = [-(-(x + (N if op == "write" else 0)) // PAGE) for x in lens]
    width, pages = max(1, max(need)), sum(need) + 3
    perm = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    st = {"table": table, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    for name in ("k", "v"):
        st[name + "_pages"] = torch.randint(0, 256, (pages, Hkv, PAGE, d // 2), generator=gen, device="cuda",
                                            dtype=torch.uint8)
        st[name + "_scales"] = torch.randint(124, 128, (pages, Hkv, d // GROUP, PAGE), generator=gen, device="cuda",
                                             dtype=torch.uint8)
    if op == "write":
        for name in ("k", "v"):
            x = torch.randn((B, Hkv, N, d // GROUP, GROUP), generator=gen, device="cuda")
            x *= torch.exp2(2 * torch.randn((B, Hkv, N, d // GROUP, 1), generator=gen, device="cuda"))
            st[name] = x.view(B, Hkv, N, d).to(torch.bfloat16)
    elif op == "attn":
        st["q"] = torch.randn((B, H, N, d), generator=gen, device="cuda").to(torch.bfloat16)
    return st


def prepare(case, seed):
    return {**_inputs(case, seed), "case": case}


# ---------------------------------------------------------------------------------------------
# plain forms


def _pairs(case, dev="cuda"):
    """First and second values of the pairs of all axes: indices into a head's d values."""
    dims = _dims(case)
    starts = [sum(dims[:i]) for i in range(len(dims))]
    if case["layout"] == "split":
        first = torch.arange(sum(dims) // 2, device=dev)
        return first, first + sum(dims) // 2
    first, second = [], []
    for s, n in zip(starts, dims):
        j = torch.arange(n // 2, device=dev)
        first.append(s + 2 * j if case["layout"] == "interleaved" else s + j)
        second.append(s + 2 * j + 1 if case["layout"] == "interleaved" else s + n // 2 + j)
    return torch.cat(first), torch.cat(second)


def _turns(case, st):
    """Cosines and sines of the pairs' angles, [1 or B, S, 1, pairs]."""
    dims = _dims(case)
    axis = torch.cat([torch.full((n // 2,), i, device="cuda") for i, n in enumerate(dims)])
    at = st["positions"] if st["positions"].dim() == 3 else st["positions"][None]
    angle = at.double()[..., axis] * st["freqs"]
    return angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]


def _turned(case, y, cos, sin):
    i, j = _pairs(case)
    a, b = y[..., i], y[..., j]
    out = y.clone()
    out[..., i] = a * cos - b * sin
    out[..., j] = b * cos + a * sin
    return out


def _hat(case, x):
    """The normed values before the weights, and the factor that norms."""
    if not case["norm"]:
        return x, None
    if case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _valid(case, st):
    """[B, S, 1, 1]: the tokens before each sequence's end."""
    s = torch.arange(case["S"], device="cuda")
    return (s < torch.tensor(_lens(case), device="cuda")[:, None])[:, :, None, None]


def _parts(case, x):
    H, Hkv = case["H"], case["Hkv"]
    return x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]


def _head_rope(case, st):
    cos, sin = _turns(case, st)
    ok = _valid(case, st)
    out = {}
    for name, x in zip("qkv", _parts(case, st["x"])):
        y = x.float()
        if name != "v":
            y, _ = _hat(case, y)
            if case["norm"]:
                y = y * st[name + "_weight"]
            if case["norm"] == "layer":
                y = y + st[name + "_bias"]
            y = _turned(case, y, cos, sin)
        out[name] = torch.where(ok, y, 0).transpose(1, 2).to(torch.bfloat16).contiguous()
    return out


def _head_rope_grad(case, st):
    cos, sin = _turns(case, st)
    ok = _valid(case, st)
    dx, out = [], {}
    for name, x in zip("qkv", _parts(case, st["x"])):
        g = torch.where(ok, st["d" + name].transpose(1, 2).float(), 0)
        if name != "v":
            g = _turned(case, g, cos, -sin)
            if case["norm"]:
                hat, r = _hat(case, x.float())
                out["d" + name + "_weight"] = torch.where(ok, g * hat, 0).sum((0, 1, 2))
                if case["norm"] == "layer":
                    out["d" + name + "_bias"] = g.sum((0, 1, 2))
                u = g * st[name + "_weight"]
                g = u - hat * (u * hat).mean(-1, keepdim=True)
                if case["norm"] == "layer":
                    g = g - u.mean(-1, keepdim=True)
                g = g * r
        dx.append(torch.where(ok, g, 0).to(torch.bfloat16))
    out["dx"] = torch.cat(dx, 2)
    return out


def _held(x):
    """The values that stand for x [..., d] in 4 bits: the least power of two with which a group's magnitudes
    stay within 7, then the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    y = x.float().unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))
    e = torch.where(m > 0, torch.where(m <= 0.875, e - 3, e - 2), -100).clamp(-100, 125)
    a = torch.ldexp(y.abs(), -e).clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.ldexp(torch.round(a / step) * step, e)
    return torch.copysign(a, y).flatten(-2).to(torch.bfloat16)


def _values(codes, scales):
    """fp32 values of codes [..., tokens, d / 2] with scales [..., d / 32, tokens]."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    x = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).flatten(-2)
    s = torch.exp2(scales.float() - 127).transpose(-1, -2)
    return (x.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def _read(case, st):
    N, d, Hkv, table = case["N"], case["d"], case["Hkv"], st["table"]
    at = case["first"] + torch.arange(N, device="cuda")[None]
    ok = at < st["lens"][:, None]
    page = table.long()[:, (at[0] // PAGE).clamp(max=table.shape[1] - 1)].clamp(min=0)
    at = at.expand_as(page)
    out = {}
    for name in ("k", "v"):
        codes = st[name + "_pages"][page, :, at % PAGE]  # [B, N, Hkv, d / 2]
        scales = st[name + "_scales"][page, :, :, at % PAGE]  # [B, N, Hkv, d / 32]
        x = _values(codes, scales.transpose(-1, -2))
        x = torch.where(ok[:, :, None, None], x, 0)
        out[name] = x.transpose(1, 2).to(torch.bfloat16).contiguous()
    return out


def _attend(case, st):
    q, table, lens = st["q"], st["table"].long().clamp(min=0), st["lens"].long()
    B, H, N, d = q.shape
    Hkv, width = case["Hkv"], table.shape[1]

    def tokens(name):
        x = _values(st[name + "_pages"][table], st[name + "_scales"][table])
        return x.transpose(1, 2).reshape(B, Hkv, width * PAGE, d)

    s = torch.matmul(q.float().view(B, Hkv, -1, d), tokens("k").transpose(-1, -2)).mul_(d ** -0.5)
    s = s.view(B, H, N, width * PAGE)
    ends = lens[:, None] - (N - 1) + torch.arange(N, device="cuda")
    pos = torch.arange(width * PAGE, device="cuda")
    s.masked_fill_(pos >= ends[:, None, :, None], -torch.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, -1, width * PAGE), tokens("v")).view(B, H, N, d) / total.clamp(min=1e-30)
    return {"out": out.to(torch.bfloat16), "lse": (m + total.log()).squeeze(-1)}


# ---------------------------------------------------------------------------------------------


def run(state):
    case, st = state["case"], state
    if own:
        return _run_own(case, st)
    if case["op"] == "rope":
        return _head_rope(case, st)
    if case["op"] == "rope_grad":
        return _head_rope_grad(case, st)
    if case["op"] == "write":
        return {"k": _held(st["k"]), "v": _held(st["v"])}
    return _read(case, st) if case["op"] == "read" else _attend(case, st)


def _run_own(case, st):
    import paper_2502_06155_amd as ta

    if case["op"] in ("rope", "rope_grad"):
        q, k, v = _parts(case, st["x"])
        how = dict(positions=st["positions"], freqs=st["freqs"], dims=_dims(case), layout=case["layout"],
                   norm=case["norm"] or None, q_weight=st["q_weight"], k_weight=st["k_weight"],
                   q_bias=st["q_bias"], k_bias=st["k_bias"], eps=EPS, lens=st["lens"])
        if case["op"] == "rope":
            return dict(zip("qkv", ta.head_rope(q, k, v, **how)))
        dx = torch.empty_like(st["x"])
        grads = ta.head_rope_grad(q, k, v, st["dq"], st["dk"], st["dv"], out=_parts(case, dx), **how)
        names = ("dq_weight", "dk_weight", "dq_bias", "dk_bias")
        return {"dx": dx, **{n: g for n, g in zip(names, grads[3:]) if g is not None}}
    cache = tuple(st[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales", "table", "lens"))
    if case["op"] == "write":
        return dict(zip("kv", ta.cache4_write(st["k"], st["v"], *cache, return_held=True)))
    if case["op"] == "read":
        return dict(zip("kv", ta.cache4_read(*cache, case["N"], first=case["first"])))
    out, lse = ta.cache4_attn(st["q"], *cache, return_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------
# 64 bits, from the definitions, one head or sequence at a time


def exact(case, seed):
    st = _inputs(case, seed)
    f64 = dict(dtype=torch.float64, device="cuda")

    def rotation():
        """The matrix-free rotation: for every value its partner, sign and pair."""
        dims, d = _dims(case), case["d"]
        partner, sign, pair = list(range(d)), [0.0] * d, [0] * d
        axis, p, start = [], 0, 0
        for a, n in enumerate(dims):
            for j in range(n // 2):
                if case["layout"] == "interleaved":
                    i0, i1 = start + 2 * j, start + 2 * j + 1
                elif case["layout"] == "halves":
                    i0, i1 = start + j, start + n // 2 + j
                else:
                    i0, i1 = p, p + sum(dims) // 2
                partner[i0], partner[i1], sign[i0], sign[i1], pair[i0], pair[i1] = i1, i0, -1.0, 1.0, p, p
                axis.append(a)
                p += 1
            start += n
        at = st["positions"] if st["positions"].dim() == 3 else st["positions"][None].expand(case["B"], -1, -1)
        angle = at.double()[..., torch.tensor(axis, device="cuda")] * st["freqs"]
        pair, sign = torch.tensor(pair, device="cuda"), torch.tensor(sign, **f64)
        cos = torch.where(sign == 0, 1.0, torch.cos(angle)[..., pair])
        return torch.tensor(partner, device="cuda"), cos, torch.sin(angle)[..., pair] * sign

    def normed(x, name):
        if not case["norm"]:
            return x, torch.ones_like(x[..., :1]), x
        c = x - x.mean(-1, keepdim=True) if case["norm"] == "layer" else x
        r = (c.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5)
        n = c * r * st[name + "_weight"].double()
        return c * r, r, n + st[name + "_bias"].double() if case["norm"] == "layer" else n

    def heads():
        """(q, k or v, head in it, head in x)."""
        at = 0
        for name, n in (("q", case["H"]), ("k", case["Hkv"]), ("v", case["Hkv"])):
            for h in range(n):
                yield name, h, at
                at += 1

    def rope():
        partner, cos, sin = rotation()
        B, S, d = case["B"], case["S"], case["d"]
        out = {n: torch.zeros((B, h, S, d), **f64) for n, h in (("q", case["H"]), ("k", case["Hkv"]), ("v", case["Hkv"]))}
        for name, h, at in heads():
            y = st["x"][:, :, at].double()
            if name != "v":
                y = normed(y, name)[2]
                y = y * cos + y[..., partner] * sin
            for b, n in enumerate(_lens(case)):
                out[name][b, h, :n] = y[b, :n]
        return out

    def rope_grad():
        partner, cos, sin = rotation()
        out = {"dx": torch.zeros(st["x"].shape, **f64)}
        for name, h, at in heads():
            g = st["d" + name][:, h].double()
            for b, n in enumerate(_lens(case)):
                g[b, n:] = 0
            if name != "v":
                g = g * cos + (g * sin)[..., partner]
                if case["norm"]:
                    hat, r, _ = normed(st["x"][:, :, at].double(), name)
                    w = "d" + name + "_weight"
                    out[w] = out.get(w, 0) + (g * hat).sum((0, 1))
                    if case["norm"] == "layer":
                        out["d" + name + "_bias"] = out.get("d" + name + "_bias", 0) + g.sum((0, 1))
                    u = g * st[name + "_weight"].double()
                    c = (u * hat).mean(-1, keepdim=True)
                    g = (u - hat * c - (u.mean(-1, keepdim=True) if case["norm"] == "layer" else 0)) * r
            out["dx"][:, :, at] = g
        return out

    def nearest():
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], **f64)
        out = {}
        for name in ("k", "v"):
            x = st[name].double().unflatten(-1, (-1, GROUP))
            # bf16 magnitudes next to 7 * 2^e differ by 0.005 in the logarithm
            e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True).clamp(min=1e-40) / 7) - 1e-6).clamp(min=-100)
            a = x.abs() / torch.exp2(e)
            between = (grid[1:] + grid[:-1]) / 2
            up = torch.bucketize(a, between, right=True)  # a tie goes up here, down below where that is even
            tie = (up > 0) & (a == between[(up - 1).clamp(min=0)]) & (up % 2 == 1)
            got = grid[up - tie.long()] * torch.exp2(e)
            out[name] = torch.where(x < 0, -got, got).flatten(-2)
        return out

    def token_values(name, b, first, last):
        """[Hkv, last - first, d] of sequence b."""
        t = torch.arange(first, last, device="cuda")
        page = st["table"][b].long()[t // PAGE]
        codes = st[name + "_pages"][page, :, t % PAGE].long()
        scales = st[name + "_scales"][page, :, :, t % PAGE].double()
        c = torch.stack([codes % 16, codes // 16], -1).flatten(-2)
        m = c % 8
        x = torch.where(m < 2, m * 0.5, (2 + m % 2).double() * torch.exp2((m // 2).double() - 2))
        x = torch.where(c >= 8, -x, x)
        return (x.unflatten(-1, (-1, GROUP)) * torch.exp2(scales - 127)[..., None]).flatten(-2).transpose(0, 1)

    def read():
        B, Hkv, N, d = (case[k] for k in ("B", "Hkv", "N", "d"))
        out = {n: torch.zeros((B, Hkv, N, d), **f64) for n in ("k", "v")}
        for b, ln in enumerate(_lens(case)):
            have = max(0, min(ln - case["first"], N))
            for n in ("k", "v"):
                out[n][b, :, :have] = token_values(n, b, case["first"], case["first"] + have)
        return out

    def over_cache():
        q = st["q"].double()
        B, H, N, d = q.shape
        out, lse = torch.zeros_like(q), torch.full((B, H, N), -torch.inf, **f64)
        for b, ln in enumerate(_lens(case)):
            k, v = (token_values(n, b, 0, ln) for n in ("k", "v"))
            for h in range(H):
                g = h * case["Hkv"] // H
                for t in range(N):
                    end = ln - (N - 1) + t
                    if end > 0:
                        s = k[g, :end] @ q[b, h, t] * d ** -0.5
                        lse[b, h, t] = torch.logsumexp(s, 0)
                        out[b, h, t] = torch.softmax(s, 0) @ v[g, :end]
        return {"out": out, "lse": lse}

    how = {"rope": rope, "rope_grad": rope_grad, "write": nearest, "read": read, "attn": over_cache}
    return how[case["op"]]()
