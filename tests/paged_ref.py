"""Rotary positions and the paged 4-bit cache by their definitions (CPU, float64).

Rotations are exact up to one rounding in float64 (a bf16 value times an fp32 table entry has
32 significant bits), so the library's results are compared bit for bit; so are codes and
scales.
"""
from __future__ import annotations

import math

import torch

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def turn(x, cs, pairs, interleaved=False, back=False):
    """x [.., D] (bf16) turned by cs [.., pairs, 2] (fp32), rounded as the library rounds."""
    y = x.double().clone()
    c, s = cs.double()[..., 0], cs.double()[..., 1]
    if back:
        s = -s
    lo = torch.arange(pairs) * (2 if interleaved else 1)
    hi = lo + (1 if interleaved else pairs)
    a, b = y[..., lo].clone(), y[..., hi].clone()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    out = y.float().bfloat16()
    out[..., 2 * pairs:] = x[..., 2 * pairs:]
    return out


def random_table(gen, rows, pairs, amplitude=1.0):
    x = torch.rand(rows, pairs, generator=gen, dtype=torch.float64) * 2 * math.pi
    return (amplitude * torch.stack([x.cos(), x.sin()], dim=-1)).float()


def scale_exp(amax: float) -> int:
    for e in range(-125, 126):
        if amax <= 6.0 * 2.0 ** e:
            return e
    return 125


def nearest_code(y):
    """Codes of float64 y, the nearest level (|y| up to and past 6), ties to the even code."""
    a = y.abs().clamp_max(6.0)
    best, far = torch.zeros(y.shape, dtype=torch.long), torch.full(y.shape, math.inf, dtype=torch.float64)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):
        d = (a - LEVELS[code]).abs()
        best = torch.where(d < far, code, best)
        far = torch.minimum(far, d)
    return best + 8 * torch.signbit(y).long()


def encode(x):
    """(codes as bytes [.., D / 2], scale bytes [.., D / 32]) of x [.., D]; the codes of 32
    channels with a NaN among them are given as -1: unspecified."""
    w = x.double().unflatten(-1, (-1, 32))
    fin = torch.where(w.isfinite(), w.abs(), 0.0).amax(dim=-1)
    uniq, inv = fin.unique(return_inverse=True)
    e = torch.tensor([scale_exp(float(u)) for u in uniq])[inv]
    code = nearest_code(torch.where(w.isnan(), 0.0, w) * torch.exp2(-e.double())[..., None])
    bad = w.isnan().any(dim=-1)
    byte = torch.where(bad, 255, e + 127)
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    codes = code[..., 0] + 16 * code[..., 1]
    return torch.where(bad.repeat_interleave(16, dim=-1), -1, codes), byte


def decode(codes, scale):
    """float64 values [.., D] of codes [.., D / 2] and scale bytes [.., D / 32]."""
    u = codes.long()
    u = torch.stack([u % 16, u // 16], dim=-1).flatten(-2)
    x = torch.tensor(LEVELS, dtype=torch.float64)[u % 8] * (1.0 - 2.0 * (u >= 8).double())
    f = torch.exp2(scale.double() - 127)
    f = torch.where(scale == 255, math.nan, f)
    return x * f.repeat_interleave(32, dim=-1)


def sequence(pool, pages, block):
    """Rows [B, H, n_table * block, x] of a pool [P, H, block, x]; rows of pages outside it: None."""
    ok = (pages >= 0) & (pages < pool.shape[0])
    rows = pool[torch.where(ok, pages, 0).long()].transpose(1, 2).flatten(2, 3)
    return rows, ok.repeat_interleave(block, dim=1)


def write(pool_codes, pool_scale, x, pages, starts, counts=None):
    """Appends x [B, H, L, D] to the pools in place; unspecified codes become -1."""
    B, _, L, _ = x.shape
    block, P = pool_codes.shape[2], pool_codes.shape[0]
    codes, scale = encode(x)
    for b in range(B):
        n = L if counts is None else max(0, min(L, counts[b]))
        for i in range(n):
            r = starts[b] + i
            if not 0 <= r < pages.shape[1] * block:
                continue
            p = int(pages[b, r // block])
            if 0 <= p < P:
                pool_codes[p, :, r % block] = codes[b, :, i]
                pool_scale[p, :, r % block] = scale[b, :, i]
