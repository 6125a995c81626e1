"""Attention over selected blocks and over an 8-bit cache in float64, from the definitions.

Everything is dense and per head: a boolean matrix says which keys a query row attends to, and the
results follow from it. Beside the results the functions give the sums that bound what rounding
weights and outputs to bf16 can do to them.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128


def widen(bits):
    """bf16 bit patterns as float64."""
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16(x):
    """Nearest bf16 bit patterns of finite numbers, ties to even. On the way through float32 what is not
    exact goes to the neighbour with an odd last bit, which no tie of bf16 has."""
    x = np.asarray(x, np.float64)
    f = x.astype(np.float32)
    u = f.view(np.uint32).astype(np.int64)
    step = np.sign(np.abs(x) - np.abs(f.astype(np.float64))).astype(np.int64)
    u = np.where(u % 2 == 0, u + step, u).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def _lens(lens, B, S):
    return [S] * B if lens is None else [min(max(int(x), 0), S) for x in lens]


def block_means(x_bits, lens=None):
    """bf16 bits of the mean of every block's valid tokens: x [B, H, S, d]."""
    x = widen(x_bits)
    B, H, S, d = x.shape
    out = np.zeros((B, H, -(-S // BLOCK), d))
    for b, n in enumerate(_lens(lens, B, S)):
        for j in range(-(-n // BLOCK)):
            out[b, :, j] = x[b, :, BLOCK * j:min(n, BLOCK * (j + 1))].mean(1)
    return to_bf16(out)


def block_lists(q_bits, means_bits, Skv, n, causal=False, sink=0, local=1, lens=None):
    """The lists [B, Hkv, NQ, n] of the n best blocks of every query block."""
    q, km = widen(q_bits), widen(means_bits)
    B, H, Sq, d = q.shape
    Hkv = km.shape[1]
    G, off, nq = H // Hkv, Skv - Sq, -(-Sq // BLOCK)
    out = np.full((B, Hkv, nq, n), -1, np.int32)
    for b, ln in enumerate(_lens(lens, B, Skv)):
        for h in range(Hkv):
            for i in range(nq):
                r1 = min(Sq, BLOCK * (i + 1), ln - off)
                if r1 <= BLOCK * i:
                    continue
                qm = widen(to_bf16(q[b, h * G:(h + 1) * G, BLOCK * i:r1].mean((0, 1))))
                score = km[b, h] @ qm
                lo, hi = (off + BLOCK * i) // BLOCK, (off + r1 - 1) // BLOCK
                able = range(min(-(-ln // BLOCK), hi + 1) if causal else -(-ln // BLOCK))
                top = hi if causal else hi + local - 1
                must = [j for j in able if j < sink or (local > 0 and lo - local < j <= top)]
                rest = sorted(set(able) - set(must), key=lambda j: (-score[j], j))
                got = sorted((must + rest)[:n])
                out[b, h, i, :len(got)] = got
    return out


def attends(lists, Sq, Skv, causal, length):
    """bool [Sq, Skv]: which keys the rows attend to, for the lists [NQ, n] of one key head."""
    off, nb = Skv - Sq, -(-Skv // BLOCK)
    m = np.zeros((Sq, Skv), bool)
    for r in range(Sq):
        if off + r >= length:
            continue
        for j in lists[r // BLOCK]:
            if 0 <= j < nb:
                m[r, BLOCK * j:min(length, BLOCK * (j + 1))] = True
        if causal:
            m[r, off + r + 1:] = False
    return m


def _softmax(s, m):
    s = np.where(m, s, -np.inf)
    top = np.where(m.any(1), s.max(1, initial=-np.inf), 0.0)
    p = np.where(m, np.exp(s - top[:, None]), 0.0)
    l = p.sum(1)
    with np.errstate(divide="ignore"):
        return p / np.where(l > 0, l, 1.0)[:, None], top + np.log(l)


def attention(q_bits, k_bits, v_bits, lists, causal=False, lens=None, scale=None):
    """(out, lse, sum of p |v|) of attention over the lists."""
    q, k, v = widen(q_bits), widen(k_bits), widen(v_bits)
    B, H, Sq, d = q.shape
    Hkv, Skv = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    out, mag, lse = np.zeros_like(q), np.zeros_like(q), np.zeros((B, H, Sq))
    for b, ln in enumerate(_lens(lens, B, Skv)):
        for h in range(H):
            g = h * Hkv // H
            m = attends(lists[b, g], Sq, Skv, causal, ln)
            used = m.any(0)
            p, lse[b, h] = _softmax(scale * (q[b, h] @ np.where(used[:, None], k[b, g], 0).T), m)
            vv = np.where(used[:, None], v[b, g], 0)
            out[b, h], mag[b, h] = p @ vv, p @ np.abs(vv)
    return out, lse, mag


def attention_backward(q_bits, k_bits, v_bits, dout_bits, lists, causal=False, lens=None, scale=None):
    """dq, dk, dv, and for each what errors can add up to: a list of (gradient, sum of |dS| times the
    other factor (of P |dout| for dv), sum of P (|dP| + |delta|) times it, sum of P E times it), E
    being |dout| times the bound 2^-8 (|out| + sum p |v|) of out's own error."""
    q, k, v, go = widen(q_bits), widen(k_bits), widen(v_bits), widen(dout_bits)
    B, H, Sq, d = q.shape
    Hkv, Skv = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    dq = [np.zeros_like(q) for _ in range(4)]
    dk = [np.zeros_like(k) for _ in range(4)]
    dv = [np.zeros_like(k) for _ in range(2)]
    for b, ln in enumerate(_lens(lens, B, Skv)):
        for h in range(H):
            g = h * Hkv // H
            m = attends(lists[b, g], Sq, Skv, causal, ln)
            used, rows = m.any(0)[:, None], m.any(1)[:, None]
            kk, vv = np.where(used, k[b, g], 0), np.where(used, v[b, g], 0)
            qq, gg = np.where(rows, q[b, h], 0), np.where(rows, go[b, h], 0)
            p, _ = _softmax(scale * (qq @ kk.T), m)
            dp, o = gg @ vv.T, p @ vv
            delta = (gg * o).sum(1, keepdims=True)
            e = (np.abs(gg) * 2.0 ** -8 * (np.abs(o) + p @ np.abs(vv))).sum(1, keepdims=True)
            ds = p * (dp - delta)
            parts = (ds, np.abs(ds), p * (np.abs(dp) + np.abs(delta)), p * e)
            for x, part in enumerate(parts):
                f = abs(scale) if x else scale
                dq[x][b, h] += f * (part @ (np.abs(kk) if x else kk))
                dk[x][b, g] += f * (part.T @ (np.abs(qq) if x else qq))
            dv[0][b, g] += p.T @ gg
            dv[1][b, g] += p.T @ np.abs(gg)
    return dq, dk, dv


# e4m3: code c (sign, 4 exponent bits, 3 mantissa bits) and its value; 0x7f and 0xff are NaN.
def e4m3_values():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c >= 128, -x, x)


def e4m3_codes(x):
    """Nearest codes, ties to the even one; infinities become the largest code, NaN stays NaN."""
    x = np.asarray(x, np.float64)
    grid = e4m3_values()[:127]
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    lo = np.clip(np.searchsorted(grid, a, side="right") - 1, 0, 125)
    below, above = a - grid[lo], grid[lo + 1] - a
    code = np.where((above < below) | ((above == below) & (lo % 2 == 1)), lo + 1, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def page_scale(x):
    """The least 2^e, -100 <= e <= 120, with which the largest finite magnitude of x is at most 448."""
    a = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = -100
    while a > 448.0 * 2.0 ** e and e < 120:
        e += 1
    return 2.0 ** e


def cache_write(k_bits, v_bits, k_pages, v_pages, k_scales, v_scales, table, lens, n_new=None):
    """Writes into the given arrays of codes (uint8) and scales."""
    values = e4m3_values()
    B, Hkv, N, d = k_bits.shape
    for bits, pages, scales, across in ((k_bits, k_pages, k_scales, False), (v_bits, v_pages, v_scales, True)):
        x = widen(bits)
        for b in range(B):
            n0 = max(int(lens[b]), 0)
            n1 = n0 + (N if n_new is None else min(max(int(n_new[b]), 0), N))
            for slot in range(n0 // BLOCK, -(-n1 // BLOCK)):
                if slot >= table.shape[1] or not 0 <= table[b, slot] < len(pages):
                    continue
                t0, t1 = max(n0, BLOCK * slot), min(n1, BLOCK * (slot + 1))
                if t1 <= t0:
                    continue
                for h in range(Hkv):
                    page = pages[table[b, slot], h]
                    page = page.T if across else page
                    new = x[b, h, t0 - n0:t1 - n0]
                    old, s0, s1 = t0 - BLOCK * slot, float(scales[table[b, slot], h]), page_scale(new)
                    if old:
                        s1 = max(s0, s1)
                        if s1 != s0:
                            page[:old] = e4m3_codes(values[page[:old]] * (s0 / s1))
                    page[old:old + t1 - t0] = e4m3_codes(new / s1)
                    scales[table[b, slot], h] = s1


def cache_attention(q_bits, k_pages, v_pages, k_scales, v_scales, table, lens, scale=None):
    """(out, lse, sum of p |v|) of the last N tokens over the cache; table [B, pages] or [B, Hkv, pages]."""
    q, values = widen(q_bits), e4m3_values()
    B, H, N, d = q.shape
    n_pages, Hkv = k_pages.shape[:2]
    scale = d ** -0.5 if scale is None else scale
    out, mag, lse = np.zeros_like(q), np.zeros_like(q), np.zeros((B, H, N))
    for b in range(B):
        for h in range(H):
            g = h * Hkv // H
            tab, ln = (table[b, g], lens[b, g]) if table.ndim == 3 else (table[b], lens[b])
            ln = min(max(int(ln), 0), BLOCK * len(tab))
            m = np.zeros((N, BLOCK * len(tab)), bool)
            kk, vv = np.zeros((BLOCK * len(tab), d)), np.zeros((BLOCK * len(tab), d))
            for i, page in enumerate(tab):
                n = min(BLOCK, ln - BLOCK * i)
                if n <= 0 or not 0 <= page < n_pages:
                    continue
                s = slice(BLOCK * i, BLOCK * i + n)
                kk[s] = values[k_pages[page, g, :n]] * float(k_scales[page, g])
                vv[s] = values[v_pages[page, g].T[:n]] * float(v_scales[page, g])
                for t in range(N):
                    m[t, BLOCK * i:min(BLOCK * i + n, max(0, ln - (N - 1) + t))] = True
            p, lse[b, h] = _softmax(scale * (q[b, h] @ kk.T), m)
            out[b, h], mag[b, h] = p @ vv, p @ np.abs(vv)
    return out, lse, mag
