"""Plain 64-bit statements of the stand-alone operators, for their tests (numpy on the CPU)."""
from __future__ import annotations

import numpy as np


def pair_axes(pairs, layout):
    """[(axis, place on the axis)] of every pair."""
    if layout == "blocks":
        return [(a, j) for a, n in enumerate(pairs) for j in range(n)]
    out, taken = [], [0] * len(pairs)
    while len(out) < sum(pairs):
        for a, n in enumerate(pairs):
            if taken[a] < n:
                out.append((a, taken[a]))
                taken[a] += 1
    return out


def rope_angles(pos, pairs, theta=10000.0, ladder="axis", layout="blocks", scale=None):
    """[tokens][pairs] angles of positions [axes][tokens]."""
    pos = np.asarray(pos, dtype=np.float64)
    scale = scale or [1.0] * len(pairs)
    cols = []
    for i, (a, j) in enumerate(pair_axes(pairs, layout)):
        e = j / pairs[a] if ladder == "axis" else i / sum(pairs)
        cols.append(pos[a] * (scale[a] * float(theta) ** -e))
    return np.stack(cols, axis=1)


def grid_positions(grids, merge, axes):
    """[axes][tokens] of packed grids (t, h, w, t0, y0, x0), token by token."""
    out = []
    for g in grids:
        t, h, w, t0, y0, x0 = tuple(g) + (0,) * (6 - len(g))
        for f in range(t):
            for by in range(0, h, merge):
                for bx in range(0, w, merge):
                    for y in range(by, by + merge):
                        for x in range(bx, bx + merge):
                            full = (t0 + f, y0 + y, x0 + x)
                            out.append(full[3 - axes:] if axes > 1 else (t0 + (f * h + y) * w + x,))
    return np.array(out, dtype=np.int64).reshape(-1, axes).T


def head_norm(x, g, b, norm, eps):
    """Norm over the last axis: (result, factor by which x - mean was multiplied, mean |x|)."""
    x = np.asarray(x, dtype=np.float64)
    if norm is None:
        return x, np.ones_like(x[..., :1]), 0.0 * x[..., :1]
    c = x - x.mean(-1, keepdims=True) if norm == "layer" else x
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    y = c * r * (1.0 if g is None else g) + (0.0 if b is None else b)
    return y, r, np.abs(x).mean(-1, keepdims=True)


def rotate(n, cos, sin, pairing):
    """n [rows][heads][d], cos and sin [rows][pairs]."""
    p = cos.shape[1]
    out = np.array(n, dtype=np.float64)
    a, b = (slice(0, p), slice(p, 2 * p)) if pairing == "halves" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    c, s = cos[:, None, :], sin[:, None, :]
    out[..., a] = n[..., a] * c - n[..., b] * s
    out[..., b] = n[..., b] * c + n[..., a] * s
    return out


def quantized(x, axis):
    """(integers, scales) of values along `axis`, all as float64: s = max|x| / 127 and x / s each rounded to fp32, then to the
    nearest integer with ties to even."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        top = np.abs(x).max(axis=axis, keepdims=True)
        s = np.where(np.isfinite(top), top / 127.0, np.nan).astype(np.float32).astype(np.float64)
        ratio = (x / np.where(s > 0, s, 1.0)).astype(np.float32).astype(np.float64)
        q = np.where(s > 0, np.clip(np.rint(ratio), -127, 127), 0.0)
    return q, s


def gelu(x):
    return 0.5 * x * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)))
