"""A cache in 4 bits, in float64 numpy: e2m1 codes, a power of two for every 32 values of a token.

Pages hold 128 tokens of every key head: codes [pages, Hkv, 128, d / 2] (two values a byte, the even one low), scales
[pages, Hkv, d / 32, 128], exponents biased by 127, 255 for NaN.
"""
from __future__ import annotations

import numpy as np

from .blocks import BLOCK, _softmax, widen

GROUP = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest(x):
    """Codes of x: the nearest magnitude, of two as near the one whose code is even, 6 for what is larger."""
    a = np.minimum(np.abs(np.asarray(x, np.float64)), 6.0)
    off = np.abs(a[..., None] - GRID)
    # (of equal distances argmin takes the first: put even codes before odd ones)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmin(off[..., order], -1)]
    return (code + 8 * np.signbit(x)).astype(np.uint8)


def exponent(x):
    """The least e, -100 <= e <= 125, with which the magnitudes of x are at most 7 * 2^e."""
    a = np.abs(x).max(initial=0.0)
    e = -100
    while a > 7.0 * 2.0 ** e and e < 125:
        e += 1
    return e


def values(codes, scales):
    """[tokens, d] of codes [tokens, d / 2] and scales [d / 32, tokens]."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    x = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    s = scales.astype(np.float64).T
    f = np.where(s == 255, np.nan, 2.0 ** (np.minimum(s, 254) - 127))
    return x * np.repeat(f, GROUP, axis=1)


def encode(x, marked):
    """(codes [d / 2], scales [d / 32]) of a token's d numbers; infinities and NaN count as zeros."""
    x = np.where(np.isfinite(x), x, 0.0)
    codes, scales = [], []
    for g in x.reshape(-1, GROUP):
        e = exponent(g)
        codes.append(nearest(g / 2.0 ** e))
        scales.append(255 if marked else e + 127)
    c = np.concatenate(codes)
    return (c[0::2] | c[1::2] << 4).astype(np.uint8), np.array(scales, np.uint8)


def write(k_bits, v_bits, k_pages, v_pages, k_scales, v_scales, table, lens, n_new=None):
    """Writes into the given arrays; returns the values that they hold for the new tokens, zeros where none was
    written."""
    B, Hkv, N, d = k_bits.shape
    held = np.zeros((2, B, Hkv, N, d))
    k, v = widen(k_bits), widen(v_bits)
    for b in range(B):
        n0 = max(int(lens[b]), 0)
        n = N if n_new is None else min(max(int(n_new[b]), 0), N)
        for t in range(n):
            slot, at = divmod(n0 + t, BLOCK)
            if slot >= table.shape[1] or not 0 <= table[b, slot] < len(k_pages):
                continue
            page = table[b, slot]
            for h in range(Hkv):
                bad = not (np.isfinite(k[b, h, t]).all() and np.isfinite(v[b, h, t]).all())
                for i, (x, pages, scales) in enumerate(((k, k_pages, k_scales), (v, v_pages, v_scales))):
                    pages[page, h, at], scales[page, h, :, at] = encode(x[b, h, t], bad and i == 0)
                    held[i, b, h, t] = values(pages[page, h, at:at + 1], scales[page, h, :, at:at + 1])[0]
    return held


def read(k_pages, v_pages, k_scales, v_scales, table, lens, N, first=0):
    B, Hkv = len(lens), k_pages.shape[1]
    out = np.zeros((2, B, Hkv, N, 2 * k_pages.shape[3]))
    for b in range(B):
        for t in range(max(0, min(N, int(lens[b]) - first))):
            slot, at = divmod(first + t, BLOCK)
            if slot >= table.shape[1] or not 0 <= table[b, slot] < len(k_pages):
                continue
            page = table[b, slot]
            for h in range(Hkv):
                out[0, b, h, t] = values(k_pages[page, h, at:at + 1], k_scales[page, h, :, at:at + 1])[0]
                out[1, b, h, t] = values(v_pages[page, h, at:at + 1], v_scales[page, h, :, at:at + 1])[0]
    return out


def attention(q_bits, k_pages, v_pages, k_scales, v_scales, table, lens, scale=None):
    """(out, lse, sum of p |v|) of the last N tokens over the cache; table [B, pages] or [B, Hkv, pages]. A key of NaN
    makes the rows that attend to it NaN, and no others."""
    q = widen(q_bits)
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
                kk[s] = values(k_pages[page, g, :n], k_scales[page, g, :, :n])
                vv[s] = values(v_pages[page, g, :n], v_scales[page, g, :, :n])
                for t in range(N):
                    m[t, BLOCK * i:min(BLOCK * i + n, max(0, ln - (N - 1) + t))] = True
            bad = np.isnan(kk).any(1)
            p, lse[b, h] = _softmax(scale * (q[b, h] @ np.where(bad[:, None], 0.0, kk).T), m)
            out[b, h], mag[b, h] = p @ vv, p @ np.abs(vv)
            for t in range(N):
                if (m[t] & bad).any():
                    out[b, h, t] = lse[b, h, t] = np.nan
    return out, lse, mag
