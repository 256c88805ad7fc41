"""The statements of ops_ref in 64 bits on the GPU, for sizes that numpy takes long for."""
from __future__ import annotations

import math

import torch


def head_norm(x, g, b, norm, eps):
    """Norm over the last axis: (result, factor by which x - mean was multiplied, mean |x|)."""
    x = x.double()
    if norm is None:
        return x, torch.ones_like(x[..., :1]), torch.zeros_like(x[..., :1])
    c = x - x.mean(-1, keepdim=True) if norm == "layer" else x
    r = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    y = c * r
    y = y if g is None else y * g.double()
    return (y if b is None else y + b.double()), r, x.abs().mean(-1, keepdim=True)


def pair_slices(p, pairing):
    return (slice(0, p), slice(p, 2 * p)) if pairing == "halves" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))


def rotate(n, table, pairing):
    """n [rows][heads][d], table [rows][pairs][2]."""
    out = n.clone()
    a, b = pair_slices(table.shape[1], pairing)
    c, s = table[:, None, :, 0].double(), table[:, None, :, 1].double()
    out[..., a], out[..., b] = n[..., a] * c - n[..., b] * s, n[..., b] * c + n[..., a] * s
    return out


def quantized(x, axis):
    """(integers, scales) along `axis`: quotients in 64 bits, rounded to 32 (the same as one rounding, 53 >= 2 * 24 + 2 bits)
    and then to the nearest integer, ties to even."""
    x = x.double()
    top = x.abs().amax(dim=axis, keepdim=True)
    s = torch.where(torch.isfinite(top), (top / 127.0).float().double(), torch.full_like(top, math.nan))
    q = torch.where(s > 0, (x / torch.where(s > 0, s, torch.ones_like(s))).float().double().round().clamp(-127.0, 127.0),
                    torch.zeros_like(x))
    return q, s


def gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))
