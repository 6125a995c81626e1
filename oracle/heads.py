"""Norms of heads, rotation by positions of several axes, and their gradients, in float64.

A row is the d values of one head of one token. It is normed (by its root mean square, or by mean and variance),
weighted, and pairs of its values are turned by position * frequency; every value belongs to one axis (time,
height, width), in stretches of dims[0], dims[1], ... values, and values behind those are not turned.
"""
from __future__ import annotations

import numpy as np


def pairs(dims, layout):
    """[(first value, second value, axis)], pair p at index p."""
    out, start, R = [], 0, sum(dims)
    for axis, n in enumerate(dims):
        for j in range(n // 2):
            if layout == "interleaved":
                out.append((start + 2 * j, start + 2 * j + 1, axis))
            elif layout == "halves":
                out.append((start + j, start + n // 2 + j, axis))
            else:
                out.append((start // 2 + j, R // 2 + start // 2 + j, axis))
        start += n
    return out


def turn(x, positions, freqs, dims, layout, back=False):
    """x [B, S, heads, d] turned by positions [B, S, axes] (back: by the angles' negatives)."""
    y = np.array(x, np.float64)
    for p, (i, j, axis) in enumerate(pairs(dims, layout)):
        a = positions[:, :, axis].astype(np.float64) * float(freqs[p]) * (-1.0 if back else 1.0)
        c, s = np.cos(a)[:, :, None], np.sin(a)[:, :, None]
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def normed(x, norm, eps):
    """(x normed, the factor), without weights."""
    x = np.asarray(x, np.float64)
    if norm is None:
        return x, np.ones(x.shape[:-1] + (1,))
    if norm == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def forward(x, norm=None, weight=None, bias=None, eps=1e-6, positions=None, freqs=None, dims=None, layout=None,
            lens=None):
    """Rows of q or k: x [B, S, heads, d] -> [B, heads, S, d]."""
    y, _ = normed(x, norm, eps)
    y = y * (1.0 if weight is None else np.asarray(weight, np.float64))
    y = y + (0.0 if bias is None else np.asarray(bias, np.float64))
    if positions is not None:
        y = turn(y, positions, freqs, dims, layout)
    if lens is not None:
        for b, n in enumerate(lens):
            y[b, max(int(n), 0):] = 0.0
    return y.transpose(0, 2, 1, 3)


def backward(x, dy, norm=None, weight=None, bias=None, eps=1e-6, positions=None, freqs=None, dims=None, layout=None,
             lens=None):
    """(dx [B, S, heads, d], dweight, dbias) for dy [B, heads, S, d]."""
    g = np.array(dy, np.float64).transpose(0, 2, 1, 3).copy()
    x = np.array(x, np.float64)
    if lens is not None:
        for b, n in enumerate(lens):
            g[b, max(int(n), 0):] = 0.0
            x[b, max(int(n), 0):] = 0.0
    if positions is not None:
        g = turn(g, positions, freqs, dims, layout, back=True)
    if norm is None:
        return g, None, None
    hat, r = normed(x, norm, eps)
    dweight, dbias = (g * hat).sum((0, 1, 2)), g.sum((0, 1, 2))
    u = g * (1.0 if weight is None else np.asarray(weight, np.float64))
    dx = u - hat * (u * hat).mean(-1, keepdims=True)
    if norm == "layer":
        dx = dx - u.mean(-1, keepdims=True)
    return dx * r, dweight, dbias
