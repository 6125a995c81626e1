"""Timed cases of attention over selected blocks and of attention over an 8-bit cache.

A block is 128 tokens. Attention over selected blocks: the keys of a block are summed up by their
mean, a query block (the G = H / Hkv heads of a group together) scores every block by its own
mean's product with that, and its rows attend to the tokens of the n best ones. The cache holds
keys and values in e4m3, 128 tokens a page, with one power-of-two scale for each page and head.

A case is a dict of plain values:
  name    (listed cases only)
  op      "lists"  block means of the keys and the lists (one token: the means are in hand)
          "fwd"    attention over the lists, and the row log-sum-exp
          "bwd"    its gradients dq, dk, dv
          "write"  N new tokens of every sequence into the cache's pages
          "cache"  attention of the last N tokens of every sequence over the cache
  B, H, Hkv, d     batch, query heads, key heads, head dim
  Sq, Skv, n       lists, fwd, bwd: query rows, keys (the queries are the last Sq positions), list length
  causal, sink, local, ragged   order, first and near blocks always kept, lengths that differ
  N, lo, hi        write, cache: new tokens, shortest and longest sequence (write: before the call)

Sizes: 720p video (3600 tokens a latent frame; 8 and 24 frames), the CogVideoX-5B head size, and
generic ones.
"""
from __future__ import annotations

import math

import torch
import torch.nn.functional as nnf

own = False

BLOCK = 128


def _sparse(op, B, H, Hkv, Sq, Skv, d, n, causal, sink, local, ragged=False, name=None):
    c = {"op": op, "B": B, "H": H, "Hkv": Hkv, "Sq": Sq, "Skv": Skv, "d": d, "n": n, "causal": causal,
         "sink": sink, "local": local, "ragged": ragged}
    return c if name is None else {"name": name, **c}


def _paged(op, B, H, Hkv, d, N, lo, hi, name=None):
    c = {"op": op, "B": B, "H": H, "Hkv": Hkv, "d": d, "N": N, "lo": lo, "hi": hi}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # Which of 256 past blocks a decoded token looks at: one call's latency.
        _sparse("lists", 4, 16, 4, 1, 32749, 128, 32, True, 1, 2, name="lists-token"),
        # The lists of a 93-frame 720p layer, one GPU's share of the heads, a tenth of the blocks.
        _sparse("lists", 1, 6, 6, 86400, 86400, 96, 68, False, 0, 1, name="lists-93f"),
        # A padded batch of short causal sequences with grouped heads: an odd length, a unit test's size.
        _sparse("fwd", 2, 6, 2, 777, 777, 64, 4, True, 1, 1, ragged=True, name="fwd-odd"),
        # The layer of lists-93f: a sparse student's forward.
        _sparse("fwd", 1, 6, 6, 86400, 86400, 96, 68, False, 0, 1, name="fwd-93f"),
        # One token of eight sequences over the blocks chosen from 32 thousand keys.
        _sparse("fwd", 8, 16, 4, 1, 32749, 128, 32, True, 1, 2, name="fwd-token"),
        # Gradients at the CogVideoX-5B head size: text and one frame and a half, short lists.
        _sparse("bwd", 1, 12, 12, 2251, 2251, 64, 6, False, 1, 1, name="bwd-odd"),
        # Gradients of a 29-frame 720p layer, all heads: the student's training step.
        _sparse("bwd", 1, 24, 24, 28800, 28800, 96, 32, False, 0, 1, name="bwd-29f"),
        # Gradients of a causal layer with shared key heads and a sink every query block keeps.
        _sparse("bwd", 1, 16, 4, 16384, 16384, 128, 24, True, 1, 2, name="bwd-causal"),
        # One new token of 32 sequences into their pages: latency.
        _paged("write", 32, 8, 8, 128, 1, 200, 30000, name="write-token"),
        # Two prompts written at once behind what is there.
        _paged("write", 2, 8, 8, 128, 8191, 0, 100, name="write-prompt"),
        # A draft of four tokens over short sequences: latency.
        _paged("cache", 3, 12, 4, 64, 4, 700, 1500, name="cache-draft"),
        # A decoding step of 32 sequences of half a thousand to 65 thousand tokens.
        _paged("cache", 32, 32, 8, 128, 1, 512, 65536, name="cache-long"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: every operator, head dim and group size, one token to
    long sequences, odd lengths, both orders, padded batches."""
    while True:
        op = rng.choice(["lists", "fwd", "fwd", "bwd", "bwd", "write", "cache", "cache"])
        d = rng.choice([64, 96, 128])
        Hkv = rng.choice([1, 2, 3, 4, 6, 8])
        B = rng.choice([1, 1, 2, 3, 4, 8])
        if op in ("write", "cache"):
            B = _log_int(rng, 1, 48)
            H = Hkv * rng.choice([1, 2, 3, 4, 8])
            N = _log_int(rng, 1, 6000) if op == "write" and rng.random() < 0.5 else rng.choice([1, 1, 1, 2, 5])
            hi = _log_int(rng, N, 50000) if op == "cache" else _log_int(rng, 1, 20000)
            lo = rng.randint(0 if op == "write" else min(N, hi), hi)
            case = _paged(op, B, H, Hkv, d, N, lo, hi)
        else:
            H = Hkv * rng.choice([1, 1, 2, 4])
            causal = rng.random() < 0.5
            Skv = _log_int(rng, 100, 40000)
            Sq = Skv
            if op != "bwd" and rng.random() < 0.3:
                Sq = rng.choice([1, 1, rng.randint(1, Skv)])
            sink, local = rng.choice([0, 1]), rng.choice([1, 2])
            n = _log_int(rng, 6, 100)
            case = _sparse(op, B, H, Hkv, Sq, Skv, d, n, causal, sink, local, ragged=rng.random() < 0.4)
        w = work(case)
        if w["flops"] <= 1.3e12 and w["bytes"] <= 8e8 and _elements(case) <= 4e9:
            return case


def _elements(case):
    """Scores that the plain form holds at once."""
    B, H = case["B"], case["H"]
    if case["op"] in ("write", "cache"):
        return B * max(case["Hkv"] * case["d"], H * case["N"]) * (case["hi"] + case["N"])
    nq, nb = _blocks(case)
    if case["op"] == "lists":
        return 4 * B * case["Hkv"] * nq * nb
    return B * nq * BLOCK * BLOCK * min(case["n"], nb) * max(H, case["Hkv"] * case["d"] // 64)


def _blocks(case):
    return -(-case["Sq"] // BLOCK), -(-case["Skv"] // BLOCK)


def _lens(case):
    """Tokens of each sequence: all of them, or with ragged from all down to half, all of the query
    rows' positions among them where there is one query row. Write and cache: from hi down to lo,
    evenly over the logarithm (cache: with the N new tokens)."""
    B = case["B"]
    if case["op"] in ("write", "cache"):
        lo, hi = case["lo"], case["hi"]
        f = [(math.log(lo + 1) * b + math.log(hi + 1) * (B - 1 - b)) / max(1, B - 1) for b in range(B)]
        return [min(hi, max(lo, round(math.exp(x)) - 1)) for x in f]
    S = case["Skv"]
    if not case["ragged"]:
        return [S] * B
    return [S - (b * S) // (2 * B) for b in range(B)]


def _listed_blocks(case):
    """(b, query block, its valid rows, first position, blocks its list holds)."""
    nq, _ = _blocks(case)
    off = case["Skv"] - case["Sq"]
    for b, ln in enumerate(_lens(case)):
        for i in range(nq):
            rows = max(0, min(BLOCK, case["Sq"] - BLOCK * i, ln - off - BLOCK * i))
            if rows:
                last = off + BLOCK * i + rows - 1
                able = (last if case["causal"] else ln - 1) // BLOCK + 1
                yield b, i, rows, off + BLOCK * i, min(case["n"], able), able


def _pairs(case):
    """Query-key pairs of one head over the batch: full blocks, but for the triangle of the query
    block's own position in causal order and for the tokens past a sequence's end."""
    lens, pairs = _lens(case), 0
    for b, _, rows, first, held, able in _listed_blocks(case):
        if case["causal"]:  # the blocks before the first row's, and the rows' own
            before = first // BLOCK
            near = able - before
            own_tokens = sum(first + r + 1 - BLOCK * before for r in range(rows))
            pairs += max(0, held - near) * BLOCK * rows + own_tokens
        else:
            pairs += held * rows * lens[b] / able
    return pairs


def work(case):
    """What the operator cannot do without: every input read once and every output written once, two
    products of 2 d operations per query-key pair forward and five in the gradients."""
    B, H, Hkv, d, op = (case[k] for k in ("B", "H", "Hkv", "d", "op"))
    if op in ("write", "cache"):
        lens = _lens(case)
        if op == "write":
            new = B * case["N"] * Hkv * d * 2
            return {"bytes": new * 3, "flops": 4.0 * new}
        tokens = sum(lens)
        pages = sum(-(-x // BLOCK) for x in lens)
        rows = B * H * case["N"]
        return {"bytes": tokens * Hkv * d * 2 + pages * Hkv * 8 + rows * (4 * d + 4),
                "flops": 4.0 * d * H * case["N"] * tokens}
    Sq, Skv, n = case["Sq"], case["Skv"], case["n"]
    nq, nb = _blocks(case)
    q, k = B * H * Sq * d * 2, B * Hkv * Skv * d * 2
    lists = B * Hkv * nq * n * 4
    if op == "lists":
        means = B * Hkv * nb * d * 2
        return {"bytes": q + (k if Sq > 1 else 0) + means + lists,
                "flops": 2.0 * B * Hkv * nq * nb * d + (q + (k if Sq > 1 else 0)) / 2}
    pairs = H * _pairs(case)
    if Sq < n * BLOCK:  # few rows reach only the listed blocks
        k = min(k, B * Hkv * nq * n * BLOCK * d * 2)
    if op == "fwd":
        return {"bytes": 2 * q + 2 * k + B * H * Sq * 4 + lists, "flops": 4.0 * d * pairs}
    return {"bytes": 4 * q + 4 * k + B * H * Sq * 4 + lists, "flops": 10.0 * d * pairs}


# ---------------------------------------------------------------------------------------------
# inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 29)


def _video(gen, B, H, S, d):
    """N(0, 1) plus half of a N(0, 1) for each 128 tokens: tokens near each other are alike."""
    nb = -(-S // BLOCK)
    x = torch.randn((B, H, nb, BLOCK, d), generator=gen, device="cuda")
    x += 0.5 * torch.randn((B, H, nb, 1, d), generator=gen, device="cuda")
    return x.view(B, H, nb * BLOCK, d)[:, :, :S].to(torch.bfloat16).contiguous()


def _gate(case, dev="cuda"):
    """able, forced: bool [B, 1, NQ, NB], and the valid rows [B, NQ] of each query block."""
    nq, nb = _blocks(case)
    lens = torch.tensor(_lens(case), device=dev)[:, None]
    off = case["Skv"] - case["Sq"]
    first = off + BLOCK * torch.arange(nq, device=dev)[None, :]
    most = (case["Sq"] - BLOCK * torch.arange(nq, device=dev)).clamp(max=BLOCK)[None, :]
    rows = torch.minimum(lens - first, most).clamp(min=0)
    last = first + rows - 1
    j = torch.arange(nb, device=dev)[None, None, :]
    able = (j * BLOCK < lens[:, :, None]) & (rows > 0)[:, :, None]
    lo, hi = (first // BLOCK)[:, :, None], (last // BLOCK)[:, :, None]
    if case["causal"]:
        able = able & (j * BLOCK <= last[:, :, None])
        near = (j > lo - case["local"]) & (j <= hi)
    else:
        near = (j > lo - case["local"]) & (j < hi + case["local"])
    forced = able & ((j < case["sink"]) | (near if case["local"] else torch.zeros_like(near)))
    return able[:, None], forced[:, None], rows


def _take(score, able, forced, n):
    """The n best able blocks, forced ones first, equal scores by index; ascending, -1 behind."""
    nb = score.shape[-1]
    score = torch.where(forced, torch.inf, score).masked_fill(~able, -torch.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n]
    got = torch.where(able.expand_as(score).gather(-1, best), best, nb)
    got = torch.sort(got, dim=-1).values
    got = torch.where(got < nb, got, -1).to(torch.int32)
    return nnf.pad(got, (0, n - got.shape[-1]), value=-1).contiguous()


def _inputs(case, seed):
    gen = _gen(seed)
    B, H, Hkv, d = (case[k] for k in ("B", "H", "Hkv", "d"))
    if case["op"] in ("write", "cache"):
        return _pages(case, gen)
    Sq, Skv = case["Sq"], case["Skv"]
    nq, nb = _blocks(case)
    st = {"q": _video(gen, B, H, Sq, d), "k": _video(gen, B, Hkv, Skv, d), "lens": None}
    if case["ragged"]:
        st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    if case["op"] == "lists":
        return st
    st["v"] = _video(gen, B, Hkv, Skv, d)
    # Lists as the score gives them: some blocks are liked by most query blocks.
    able, forced, _ = _gate(case)
    score = torch.randn((B, Hkv, nq, nb), generator=gen, device="cuda")
    score += torch.randn((B, Hkv, 1, nb), generator=gen, device="cuda")
    st["lists"] = _take(score, able, forced, case["n"])
    if case["op"] == "bwd":
        st["dout"] = torch.randn((B, H, Sq, d), generator=gen, device="cuda").to(torch.bfloat16)
    return st


def _pages(case, gen):
    """A cache whose sequences hold their tokens, pages in random places, and the new tokens (write)
    or the queries (cache). Scales: as writing blocks of such tokens gives them."""
    B, H, Hkv, d, N = (case[k] for k in ("B", "H", "Hkv", "d", "N"))
    lens = _lens(case)
    total = [x + (N if case["op"] == "write" else 0) for x in lens]
    need = [-(-x // BLOCK) for x in total]
    width, pages = max(1, max(need)), sum(need) + 3
    perm = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    st = {"table": table, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    for name, shape in (("k", (pages, Hkv, BLOCK, d)), ("v", (pages, Hkv, d, BLOCK))):
        e = torch.randint(-7, -4, (pages, Hkv), generator=gen, device="cuda")
        x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
        st[name + "_scale"] = torch.exp2(e.float())
        x = x / st[name + "_scale"][:, :, None, None]
        st[name + "_pages"] = x.clamp(-448, 448).to(torch.float8_e4m3fn)
    if case["op"] == "write":
        st["k"] = torch.randn((B, Hkv, N, d), generator=gen, device="cuda").to(torch.bfloat16)
        st["v"] = torch.randn((B, Hkv, N, d), generator=gen, device="cuda").to(torch.bfloat16)
    else:
        st["q"] = torch.randn((B, H, N, d), generator=gen, device="cuda").to(torch.bfloat16)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["op"] == "lists" and case["Sq"] == 1:  # a decoding program keeps its blocks' means
        st["means"] = _means(st["k"], st["lens"])
    if case["op"] == "bwd":  # the step's forward has run
        st["out"], st["lse"] = _attend(case, st)
    return st


# ---------------------------------------------------------------------------------------------
# plain forms


def _means(x, lens):
    """bf16 mean of each block's valid tokens; sums of bf16 values are exact in 64 bits."""
    B, H, S, d = x.shape
    nb = -(-S // BLOCK)
    x = nnf.pad(x, (0, 0, 0, nb * BLOCK - S)).view(B, H, nb, BLOCK, d)
    pos = torch.arange(nb * BLOCK, device=x.device).view(1, 1, nb, BLOCK, 1)
    ln = torch.full((B,), S, device=x.device) if lens is None else lens
    ok = pos < ln.view(B, 1, 1, 1, 1)
    total = torch.where(ok, x, 0).sum(3, dtype=torch.float64)
    return (total / ok.sum(3).clamp(min=1)).to(torch.bfloat16)


def _query_means(case, q, rows):
    B, H, Sq, d = q.shape
    Hkv = case["Hkv"]
    G, (nq, _) = H // Hkv, _blocks(case)
    x = nnf.pad(q, (0, 0, 0, nq * BLOCK - Sq)).view(B, Hkv, G, nq, BLOCK, d)
    ok = torch.arange(BLOCK, device=q.device) < rows[:, :, None]
    total = torch.where(ok.view(B, 1, 1, nq, BLOCK, 1), x, 0).sum((2, 4), dtype=torch.float64)
    return (total / (G * rows).clamp(min=1).view(B, 1, nq, 1)).to(torch.bfloat16)


def _choose(case, st):
    means = st["means"] if "means" in st else _means(st["k"], st["lens"])
    able, forced, rows = _gate(case)
    qm = _query_means(case, st["q"], rows)
    score = torch.matmul(qm.double(), means.double().transpose(-1, -2))
    return {"means": means, "lists": _take(score, able, forced, case["n"])}


def _rows(x, Hkv):
    """[B, H, S, ...] as [B, Hkv, NQ, G * 128, ...]: a query block's rows, the group's heads together."""
    B, H, S, *rest = x.shape
    nq = -(-S // BLOCK)
    x = nnf.pad(x, (0, 0) * len(rest) + (0, nq * BLOCK - S)).view(B, Hkv, H // Hkv, nq, BLOCK, *rest)
    return x.transpose(2, 3).reshape(B, Hkv, nq, H // Hkv * BLOCK, *rest)


def _unrows(x, H, S):
    B, Hkv, nq, _, *rest = x.shape
    x = x.view(B, Hkv, nq, H // Hkv, BLOCK, *rest).transpose(2, 3)
    return x.reshape(B, H, nq * BLOCK, *rest)[:, :, :S].contiguous()


def _gathered(x, at):
    """The tokens of the blocks `at` [B, Hkv, NQ, n] of x [B, Hkv, S, d]: [B, Hkv, NQ, n * 128, d]."""
    B, Hkv, S, d = x.shape
    nb = -(-S // BLOCK)
    x = nnf.pad(x.float(), (0, 0, 0, nb * BLOCK - S)).view(B, Hkv, nb, BLOCK * d)
    nq, n = at.shape[2:]
    x = x.gather(2, at.view(B, Hkv, nq * n, 1).expand(-1, -1, -1, BLOCK * d))
    return x.view(B, Hkv, nq, n * BLOCK, d)


def _scores(case, st):
    """Scaled scores [B, Hkv, NQ, G * 128, n * 128] with -inf where a row does not attend, and the
    list entries as valid block indices."""
    lists, dev = st["lists"], st["q"].device
    B, Hkv, nq, n = lists.shape
    G = case["H"] // Hkv
    at = lists.clamp(min=0).long()
    qf = _rows(st["q"].float(), Hkv)
    s = torch.matmul(qf, _gathered(st["k"], at).transpose(-1, -2)).mul_(case["d"] ** -0.5)
    kpos = (at[..., None] * BLOCK + torch.arange(BLOCK, device=dev)).view(B, Hkv, nq, 1, n * BLOCK)
    row = torch.arange(nq * BLOCK, device=dev).view(nq, 1, BLOCK).expand(nq, G, BLOCK).reshape(nq, G * BLOCK, 1)
    qpos = case["Skv"] - case["Sq"] + row
    ln = torch.tensor(_lens(case), device=dev).view(B, 1, 1, 1, 1)
    here = (lists >= 0)[..., None].expand(B, Hkv, nq, n, BLOCK).reshape(kpos.shape) & (kpos < ln)
    s.masked_fill_(~here, -torch.inf)
    s.masked_fill_((qpos >= ln) | (row >= case["Sq"]), -torch.inf)
    if case["causal"]:
        s.masked_fill_(kpos > qpos, -torch.inf)
    return s, at


def _attend(case, st):
    s, at = _scores(case, st)
    m = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _gathered(st["v"], at)) / total.clamp(min=1e-30)
    lse = (m + total.log()).squeeze(-1)
    H, Sq = case["H"], case["Sq"]
    return _unrows(out, H, Sq).to(torch.bfloat16), _unrows(lse, H, Sq)


def _gradients(case, st):
    H, Hkv, Sq, Skv, d = (case[k] for k in ("H", "Hkv", "Sq", "Skv", "d"))
    s, at = _scores(case, st)
    lse = _rows(st["lse"], Hkv)[..., None]
    p = s.sub_(lse.clamp(min=-1e30)).exp_()
    qf, go = _rows(st["q"].float(), Hkv), _rows(st["dout"].float(), Hkv)
    delta = (go * _rows(st["out"].float(), Hkv)).sum(-1, keepdim=True)
    kg, vg = _gathered(st["k"], at), _gathered(st["v"], at)
    dv = torch.matmul(p.transpose(-1, -2), go)
    ds = torch.matmul(go, vg.transpose(-1, -2)).sub_(delta).mul_(p)
    dq = torch.matmul(ds, kg).mul_(d ** -0.5)
    dk = torch.matmul(ds.transpose(-1, -2), qf).mul_(d ** -0.5)
    B, nb = at.shape[0], -(-Skv // BLOCK)
    flat = (torch.arange(B * Hkv, device=at.device).view(B, Hkv, 1, 1) * nb + at).view(-1)
    sums = [torch.zeros((B * Hkv * nb, BLOCK * d), device=at.device).index_add_(0, flat, x.view(-1, BLOCK * d))
            for x in (dk, dv)]
    dk, dv = (x.view(B, Hkv, nb * BLOCK, d)[:, :, :Skv].to(torch.bfloat16).contiguous() for x in sums)
    return {"dq": _unrows(dq, H, Sq).to(torch.bfloat16), "dk": dk, "dv": dv}


def _write(case, st):
    """New tokens behind each sequence's: the page's scale becomes the larger of its own (if it held
    tokens) and the least power of two with which the new tokens stay within 448; its old tokens are
    rounded again where that moved it."""
    B, Hkv, N, d = st["k"].shape
    dev = st["k"].device
    lens, table = st["lens"].long(), st["table"]
    most = (BLOCK - 1 + N + BLOCK - 1) // BLOCK  # pages that N tokens can touch
    page0 = lens // BLOCK
    slot = page0[:, None] + torch.arange(most, device=dev)
    pos = slot[:, :, None] * BLOCK + torch.arange(BLOCK, device=dev)
    old = (pos < lens[:, None, None])[:, :, None, :, None]
    token = pos - lens[:, None, None]
    new = ((token >= 0) & (token < N))[:, :, None, :, None]
    touched = new.any(3)[:, :, 0, 0]
    page = table.long().gather(1, slot.clamp(max=table.shape[1] - 1))[touched]
    out = {}
    for name in ("k", "v"):
        codes, scale = st[name + "_pages"], st[name + "_scale"]
        x = st[name].float().gather(2, token.clamp(0, N - 1).view(B, 1, -1, 1).expand(B, Hkv, -1, d))
        x = x.view(B, Hkv, most, BLOCK, d).transpose(1, 2)[touched]
        have, add = old.expand(-1, -1, Hkv, -1, d)[touched], new.expand(-1, -1, Hkv, -1, d)[touched]
        raw = codes.view(torch.uint8)  # indexing moves bytes
        c0, s0 = raw[page].view(codes.dtype).float(), scale[page]
        if name == "v":
            c0 = c0.transpose(-1, -2)
        m, e = torch.frexp(torch.where(add, x, 0).abs().amax((-1, -2)))
        e = torch.where(m > 0, torch.where(m <= 0.875, e - 9, e - 8), -100).clamp(-100, 120)
        s1 = torch.exp2(e.float())
        s1 = torch.where(have.any(-1).any(-1), torch.maximum(s0, s1), s1)
        y = torch.where(have, c0 * (s0 / s1)[:, :, None, None], x / s1[:, :, None, None])
        y = torch.where(have | add, y, c0).clamp(-448, 448)
        y = (y.transpose(-1, -2) if name == "v" else y).contiguous()
        raw[page] = y.to(codes.dtype).view(torch.uint8)
        scale[page] = s1
        out[name + "_pages"], out[name + "_scale"] = codes, scale
    return out


def _attend_cache(case, st):
    q, table, lens = st["q"], st["table"].long().clamp(min=0), st["lens"].long()
    B, H, N, d = q.shape
    Hkv, width = case["Hkv"], table.shape[1]
    k = st["k_pages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    k = (k * st["k_scale"][table][..., None, None]).transpose(1, 2).reshape(B, Hkv, width * BLOCK, d)
    s = torch.matmul(q.float().view(B, Hkv, -1, d), k.transpose(-1, -2)).mul_(d ** -0.5)
    del k
    s = s.view(B, H, N, width * BLOCK)
    ends = lens[:, None] - (N - 1) + torch.arange(N, device=q.device)
    pos = torch.arange(width * BLOCK, device=q.device)
    s.masked_fill_(pos >= ends[:, None, :, None], -torch.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = st["v_pages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()
    v = (v * st["v_scale"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, Hkv, width * BLOCK, d)
    v.masked_fill_((pos >= lens[:, None])[:, None, :, None], 0)
    out = torch.matmul(p.view(B, Hkv, -1, width * BLOCK), v).view(B, H, N, d) / total.clamp(min=1e-30)
    return {"out": out.to(torch.bfloat16), "lse": (m + total.log()).squeeze(-1)}


# ---------------------------------------------------------------------------------------------


def run(state):
    case, st = state["case"], state
    if own:
        return _run_own(case, st)
    if case["op"] == "lists":
        return _choose(case, st)
    if case["op"] == "fwd":
        out, lse = _attend(case, st)
        return {"out": out, "lse": lse}
    if case["op"] == "bwd":
        return _gradients(case, st)
    return _write(case, st) if case["op"] == "write" else _attend_cache(case, st)


def _run_own(case, st):
    import paper_2502_06155_amd as ta

    if case["op"] == "lists":
        means = st["means"] if "means" in st else ta.block_means(st["k"], lens=st["lens"])
        lists = ta.block_lists(st["q"], means, case["Skv"], case["n"], causal=case["causal"], sink=case["sink"],
                               local=case["local"], lens=st["lens"])
        return {"means": means, "lists": lists}
    if case["op"] == "fwd":
        out, lse = ta.block_attn(st["q"], st["k"], st["v"], st["lists"], causal=case["causal"], lens=st["lens"],
                                 return_lse=True)
        return {"out": out, "lse": lse}
    if case["op"] == "bwd":
        dq, dk, dv = ta.block_attn_grad(st["q"], st["k"], st["v"], st["lists"], st["out"], st["dout"], st["lse"],
                                        causal=case["causal"], lens=st["lens"])
        return {"dq": dq, "dk": dk, "dv": dv}
    cache = (st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["table"], st["lens"])
    if case["op"] == "write":
        ta.cache_write(st["k"], st["v"], *cache)
        return {k: st[k] for k in ("k_pages", "k_scale", "v_pages", "v_scale")}
    out, lse = ta.cache_attn(st["q"], *cache, return_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------
# 64 bits, from the definitions, one sequence or list at a time


def exact(case, seed):
    def lists_of(st):
        B, H, Hkv, Sq, Skv, d, n = (case[k] for k in ("B", "H", "Hkv", "Sq", "Skv", "d", "n"))
        nq, nb = _blocks(case)
        off, G = Skv - Sq, H // Hkv
        means = torch.zeros((B, Hkv, nb, d), dtype=torch.float64, device="cuda")
        lists = torch.full((B, Hkv, nq, n), -1, dtype=torch.int32)
        for b, ln in enumerate(_lens(case)):
            for j in range(-(-ln // BLOCK)):
                means[b, :, j] = st["k"][b, :, BLOCK * j:min(ln, BLOCK * (j + 1))].double().mean(1)
            km = means[b].to(torch.bfloat16).double()
            for i in range(nq):
                r0, r1 = BLOCK * i, min(Sq, BLOCK * (i + 1), ln - off)
                if r1 <= r0:
                    continue
                q = st["q"][b, :, r0:r1].double().reshape(Hkv, G * (r1 - r0), d)
                qm = q.mean(1).to(torch.bfloat16).double()
                score = (km * qm[:, None, :]).sum(-1).cpu()
                lo, hi = (off + r0) // BLOCK, (off + r1 - 1) // BLOCK
                able = range(hi + 1 if case["causal"] else -(-ln // BLOCK))
                top = hi if case["causal"] else hi + case["local"] - 1
                for h in range(Hkv):
                    row = score[h].tolist()
                    must = [j for j in able if j < case["sink"] or (case["local"] and lo - case["local"] < j <= top)]
                    rest = sorted(set(able) - set(must), key=lambda j: (-row[j], j))
                    got = sorted((must + rest)[:n])
                    lists[b, h, i, :len(got)] = torch.tensor(got, dtype=torch.int32)
        return {"means": means, "lists": lists}

    def attention(st):
        B, H, Hkv, Sq, Skv, d = (case[k] for k in ("B", "H", "Hkv", "Sq", "Skv", "d"))
        G, off, scale = H // Hkv, Skv - Sq, d ** -0.5
        lists = st["lists"].tolist()
        f64 = dict(dtype=torch.float64, device="cuda")
        out, lse = torch.zeros((B, H, Sq, d), **f64), torch.full((B, H, Sq), -torch.inf, **f64)
        bwd = case["op"] == "bwd"
        if bwd:
            dq, dk, dv = torch.zeros((B, H, Sq, d), **f64), *(torch.zeros((B, Hkv, Skv, d), **f64) for _ in range(2))
        for b, ln in enumerate(_lens(case)):
            for h in range(Hkv):
                k, v = st["k"][b, h].double(), st["v"][b, h].double()
                q = st["q"][b, h * G:(h + 1) * G].double()
                go = st["dout"][b, h * G:(h + 1) * G].double() if bwd else None
                for i, blocks in enumerate(lists[b][h]):
                    r0, r1 = BLOCK * i, min(Sq, BLOCK * (i + 1), ln - off)
                    blocks = [j for j in blocks if j >= 0]
                    if r1 <= r0 or not blocks:
                        continue
                    t = (torch.tensor(blocks, device="cuda")[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).view(-1)
                    t = t[t < ln]
                    kk, vv = k[t], v[t]
                    x = q[:, r0:r1].reshape(-1, d)
                    s = (x @ kk.t()).view(G, r1 - r0, -1) * scale
                    if case["causal"]:
                        s.masked_fill_(t > torch.arange(off + r0, off + r1, device="cuda")[:, None], -torch.inf)
                    z = torch.logsumexp(s, -1)
                    p = torch.exp(s - z.clamp(min=-1e300)[..., None]).view(G * (r1 - r0), -1)
                    o = p @ vv
                    out[b, h * G:(h + 1) * G, r0:r1] = o.view(G, r1 - r0, d)
                    lse[b, h * G:(h + 1) * G, r0:r1] = z
                    if bwd:
                        g = go[:, r0:r1].reshape(-1, d)
                        ds = p * (g @ vv.t() - (g * o).sum(1, keepdim=True))
                        dq[b, h * G:(h + 1) * G, r0:r1] = (ds @ kk).view(G, r1 - r0, d) * scale
                        dk[b, h].index_add_(0, t, ds.t() @ x, alpha=scale)
                        dv[b, h].index_add_(0, t, p.t() @ g)
        return {"dq": dq, "dk": dk, "dv": dv} if bwd else {"out": out, "lse": lse}

    def written(st):
        """Codes before their last rounding, as numbers, and the scales."""
        B, Hkv, N, d = st["k"].shape
        if B * Hkv * (N // BLOCK + 2) > 20000:
            return None
        out = {}
        for name in ("k", "v"):
            codes, scale = st[name + "_pages"].double(), st[name + "_scale"].double()
            codes = codes.transpose(-1, -2) if name == "v" else codes
            codes = codes.contiguous()
            for b, ln in enumerate(_lens(case)):
                for slot in range(ln // BLOCK, (ln + N - 1) // BLOCK + 1):
                    page = int(st["table"][b, slot])
                    t0, t1 = max(ln, BLOCK * slot), min(ln + N, BLOCK * (slot + 1))
                    x = st[name][b, :, t0 - ln:t1 - ln].double()
                    amax = x.abs().amax((1, 2)).tolist()
                    for h in range(Hkv):
                        e = -100
                        while amax[h] > 448 * 2.0 ** e:
                            e += 1
                        s1, s0 = 2.0 ** e, float(scale[page, h])
                        if t0 > BLOCK * slot:
                            s1 = max(s0, s1)
                            codes[page, h, :t0 - BLOCK * slot] *= s0 / s1
                        codes[page, h, t0 - BLOCK * slot:t1 - BLOCK * slot] = x[h] / s1
                        scale[page, h] = s1
            out[name + "_pages"] = codes.transpose(-1, -2).contiguous() if name == "v" else codes
            out[name + "_scale"] = scale
        return out

    def over_cache(st):
        q = st["q"].double()
        B, H, N, d = q.shape
        Hkv = case["Hkv"]
        out = torch.zeros_like(q)
        lse = torch.full((B, H, N), -torch.inf, dtype=torch.float64, device="cuda")
        for b, ln in enumerate(_lens(case)):
            pages = st["table"][b, :-(-ln // BLOCK)].long()
            k, v = (st[x + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()
                    * st[x + "_scale"][pages].double()[..., None, None] for x in ("k", "v"))
            for h in range(H):
                kk = k[:, h * Hkv // H].reshape(-1, d)[:ln]
                vv = v[:, h * Hkv // H].transpose(1, 2).reshape(-1, d)[:ln]
                for t in range(N):
                    end = ln - (N - 1) + t
                    if end > 0:
                        s = kk[:end] @ q[b, h, t] * d ** -0.5
                        lse[b, h, t] = torch.logsumexp(s, 0)
                        out[b, h, t] = torch.softmax(s, 0) @ vv[:end]
        return {"out": out, "lse": lse}

    how = {"lists": lists_of, "fwd": attention, "bwd": attention, "write": written, "cache": over_cache}
    return how[case["op"]](_inputs(case, seed))
