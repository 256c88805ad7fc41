"""Plain statements of the cache in 8 bits and of the attention operators, in 64 bits, for their tests (torch, on the device of
the inputs)."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24  # half a step of fp32
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def f32(x):
    return x.float().double()


class Held:
    """Keys or values in 8 bits: whole numbers [blocks][block][heads][d] and scales [blocks][heads], written row by row."""

    def __init__(self, blocks, heads, d, block=16):
        self.q = torch.zeros(blocks, block, heads, d, dtype=torch.float64)
        self.s = torch.zeros(blocks, heads, dtype=torch.float64)
        self.blocks, self.block = blocks, block

    def write(self, x, slots, begin=False):
        x, B = x.double().cpu(), self.block
        groups = {}
        for r, sl in enumerate(slots):
            if 0 <= sl < self.blocks * B:
                groups.setdefault(sl // B, {})[sl % B] = r  # the last row of a slot
        for b, rows in groups.items():
            anew = len(rows) == B or (begin and 0 in rows)
            old = torch.zeros_like(self.s[b]) if anew else self.s[b].clone()
            if anew:
                self.q[b] = 0
            new = x[list(rows.values())]  # [rows][heads][d]
            top = new.abs().amax(dim=(0, 2))
            fresh = torch.where(torch.isfinite(top), f32(top / 127.0), torch.full_like(top, math.nan))
            s = torch.where(old.isnan() | fresh.isnan(), torch.full_like(old, math.nan), torch.maximum(old, fresh))
            live = s > 0
            safe = torch.where(live, s, torch.ones_like(s))
            ratio = torch.where(live, f32(old / safe), torch.zeros_like(s))
            ratio = torch.where(s == old, torch.where(live, torch.ones_like(s), torch.zeros_like(s)), ratio)
            self.q[b] = torch.where(live[None, :, None], f32(self.q[b] * ratio[None, :, None]).round(), 0.0)
            for t, r in rows.items():
                q = f32(x[r] / safe[:, None]).round().clamp(-127, 127)
                self.q[b, t] = torch.where(live[:, None], q, torch.zeros_like(q))
            self.s[b] = s

    def values(self, dtype=torch.float32):
        """[blocks * block][heads][d]: q * s in fp32, rounded to dtype."""
        v = f32(self.q * self.s[:, None, :, None]).float().to(dtype)
        return v.reshape(-1, *v.shape[2:])

    def exact(self):
        v = self.q * self.s[:, None, :, None]
        return v.reshape(-1, *v.shape[2:])


def visible(nq, nk, causal=True, window=0, sinks=0, device="cpu"):
    p = torch.arange(nk - nq, nk, device=device)[:, None]
    j = torch.arange(nk, device=device)[None, :]
    see = j <= p if causal else torch.ones(nq, nk, dtype=torch.bool, device=device)
    if window:
        see = see & (((p - j).abs() < window) | (j < sinks))
    return see


def attention(q, k, v, see, scale=None):
    """(out, bound without the output's rounding) of one sequence: q [nq][hq][d], k and v [nk][hk][d], see [nq][nk]; keys and
    values that a row does not see do not count.

    Bound.  A score is a sum of d products (fp32 queries over the cache: 3 d) of exact factors or of ones rounded below, each
    step of the sum off by a step of fp32 (2 u of the terms' magnitudes), then times two factors (2 u) and less the maximum (u
    of the difference).  With e_j the score's error in units of ln, a weight is off by e_j + 4 u (power of 2) of itself, the
    maximum's own error cancels, and a weight divided by the sum of weights by 2 max e + 8 u.  Sums of nk terms are off by 2
    nk u, the joins of at most nk / 32 + 64 partial sums by 6 u each.  With bf16 each weight is rounded to bf16 for its product
    (2^-8); over the cache it is first multiplied by the scale (u)."""
    nq, hq, d = q.shape
    nk, hk = k.shape[:2]
    scale = d ** -0.5 if scale is None else scale
    q64, k64, v64 = q.double(), k.double(), v.double()
    out = torch.zeros(nq, hq, d, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    for h in range(hq):
        kh, vh = k64[:, h * hk // hq], v64[:, h * hk // hq]
        x = (q64[:, h] @ kh.t().contiguous()) * scale
        mag = (q64[:, h].abs() @ kh.abs().t().contiguous()) * scale
        x = torch.where(see, x, torch.full_like(x, -math.inf))
        mag = torch.where(see, mag, torch.zeros_like(mag))
        top = x.amax(-1, keepdim=True) if nk else torch.full((nq, 1), -math.inf, dtype=torch.float64, device=q.device)
        there = see.any(-1, keepdim=True)
        p = torch.where(see, torch.exp(x - torch.where(there, top, torch.zeros_like(top))), torch.zeros_like(x))
        total = p.sum(-1, keepdim=True)
        p = torch.where(there, p / torch.where(there, total, torch.ones_like(total)), torch.zeros_like(p))
        spread = torch.where(see, (top - x).abs(), torch.zeros_like(x))
        e = (2 * 3 * d + 3) * U * mag + 3 * U * torch.where(see, x.abs(), torch.zeros_like(x)) + 2 * U * spread
        e = torch.where(p > 2.0 ** -60, e, torch.zeros_like(e)).amax(-1, keepdim=True) if nk else 0.0
        rel = 2 * e + (2 * nk + 6 * (nk / 32 + 64) + 32) * U + (HALF[q.dtype] if q.dtype == torch.bfloat16 else 0.0)
        seen = see.any(0)[:, None]
        vz = torch.where(seen, vh, torch.zeros_like(vh))
        w = p @ vz.abs()
        out[:, h] = p @ vz
        bound[:, h] = rel * w
    return out, bound


def check(got, want, bound):
    """got against the 64-bit result: the bound plus one rounding to got's type."""
    d = (got.double() - want).abs()
    limit = bound + HALF[got.dtype] * (want.abs() + bound) + 1e-30
    bad = ~(d <= limit)
    assert not bad.any(), ((d / limit)[bad].max(), bad.sum(), bad.nonzero()[:4].tolist())
