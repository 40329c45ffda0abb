"""Float64 references (CPU, plain torch) for the attention gradients and the 8-bit
cache, with the error bounds that the library's arithmetic is held to.

A rounding to bf16 is off by at most U = 2^-8 of the value.  Everything else in the
kernels is fp32, whose errors (sums of a few thousand terms, the logits, exp2) are
bounded by SLACK of the same sums of magnitudes: 2^-4 of a bf16 rounding, i.e. 2^-12
relative, against about 2^-13 for 2,000 fp32 additions in a row.
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -8
SLACK = 1 + 2.0 ** -4
TINY = 1e-30


def random_lists(gen, B, H, n_q, n_k, density, kind="random"):
    """Nested [B][H][n_q] ascending lists."""
    out = []
    for _ in range(B):
        heads = []
        for h in range(H):
            rows = []
            for i in range(n_q):
                if kind == "full":
                    m = list(range(n_k))
                elif kind == "one":
                    m = [int(torch.randint(0, n_k, (1,), generator=gen))]
                else:
                    m = torch.nonzero(torch.rand(n_k, generator=gen) < density).flatten().tolist()
                if kind == "holes" and i % 3 == 1:
                    m = []
                rows.append(m)
            heads.append(rows)
        out.append(heads)
    return out


def visible(lists_h, Lq, Lk, block):
    """[Lq, Lk] mask of one head's lists (None: everything)."""
    if lists_h is None:
        return torch.ones(Lq, Lk, dtype=torch.bool)
    m = torch.zeros(Lq, Lk, dtype=torch.bool)
    for i, row in enumerate(lists_h):
        for j in row:
            m[i * block:(i + 1) * block, j * block:(j + 1) * block] = True
    return m


def forward(q, k, v, mask, scale):
    """(o, lse, p) of one head in float64; a row without keys gets 0, -inf, 0."""
    s = (q @ k.t()) * scale
    s = s.masked_fill(~mask, -math.inf)
    m = s.amax(dim=1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=s.dtype,
                                                                       device=s.device)
    m = m.masked_fill(m == -math.inf, 0.0)
    e = (s - m).exp()
    l = e.sum(dim=1, keepdim=True)
    p = e / l.clamp_min(1.0)
    return p @ v, (m + l.log())[:, 0], p


def backward(q, k, v, mask, scale, do, dlse=None):
    """dq, dk, dv of one head and the largest error that each element may have when o
    is the reference rounded to bf16."""
    o, _, p = forward(q, k, v, mask, scale)
    delta = (do * o).sum(dim=1, keepdim=True)
    if dlse is not None:
        delta = delta - dlse[:, None]
    g = do @ v.t() - delta
    ds = p * g
    dq, dk, dv = scale * ds @ k, scale * ds.t() @ q, p.t() @ do
    # delta is taken from the rounded o; dS and P are rounded once as operands; dP and
    # delta are fp32 sums of terms that may cancel
    err_delta = U * (do.abs() * o.abs()).sum(dim=1, keepdim=True)
    fp32 = (do.abs() @ v.abs().t() + (do.abs() * o.abs()).sum(dim=1, keepdim=True)) * U * 2.0 ** -8
    err_ds = p * (U * g.abs() + err_delta + fp32)
    tol = (scale * err_ds @ k.abs() + U * dq.abs(), scale * err_ds.t() @ q.abs() + U * dk.abs(),
           U * (p.t() @ do.abs()) + U * dv.abs())
    return (dq, dk, dv), tuple(t * SLACK + TINY for t in tol)


def forward_tol(q, k, v, mask, scale):
    """o, lse of one head and the largest error of each element: P rounded to bf16, O
    normalised by the sum of the rounded weights, O rounded to bf16; lse in fp32."""
    o, lse, p = forward(q, k, v, mask, scale)
    tol_o = (2 * U * (p @ v.abs()) + U * o.abs()) * SLACK + TINY
    D = q.shape[1]
    mag = (q.abs() @ k.abs().t()).amax(dim=1) * scale if k.shape[0] else torch.zeros(q.shape[0], dtype=q.dtype,
                                                                                          device=q.device)
    tol_lse = (D + 8) * 2.0 ** -24 * mag + 2.0 ** -20 * (1 + lse.abs().nan_to_num(posinf=0.0))
    return o, lse, tol_o, tol_lse


# ---- e4m3 with a power-of-two scale
def e4m3_values():
    """The value of every code, float64 [256]."""
    v = []
    for c in range(256):
        s, e, m = c >> 7, c >> 3 & 15, c & 7
        x = math.nan if e == 15 and m == 7 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        v.append(-x if s else x)
    return torch.tensor(v, dtype=torch.float64)


def e4m3_round(x):
    """The nearest e4m3 value, ties to the even code; infinities saturate, NaN stays."""
    grid = e4m3_values()[:127]
    a = x.abs().clamp_max(448.0)
    hi = torch.searchsorted(grid, a.nan_to_num(0.0)).clamp(1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return torch.where(x.isnan(), x, torch.copysign(grid[pick], x))


def scale_exp(amax: float) -> int:
    for e in range(-117, 121):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return 120


class RefCache:
    """The cache's definition, one block at a time (float64 values of the codes)."""

    def __init__(self, B, H, cap, D, block, codes, scale):
        self.block, self.cap = block, cap
        self.codes = codes.clone()       # float64 [B, H, cap, D]
        self.scale = scale.clone()       # int64 bytes [B, H, n]

    def write(self, x, starts, counts=None):
        B, H, L, _ = x.shape
        b = self.block
        for i in range(B):
            n = L if counts is None else max(0, min(L, counts[i]))
            lo, end = max(0, starts[i]), min(self.cap, starts[i] + n)
            for h in range(H):
                for j in range(lo // b, -(-end // b) if end > lo else 0):
                    r0, r1 = max(lo, j * b), min(end, (j + 1) * b)
                    new = x[i, h, r0 - starts[i]: r1 - starts[i]]
                    fin = new[new.isfinite()].abs()
                    e = scale_exp(float(fin.max()) if fin.numel() else 0.0)
                    if r0 > j * b:
                        held = min(120, max(-117, int(self.scale[i, h, j]) - 127))
                        if held < e:
                            old = self.codes[i, h, j * b: r0]
                            self.codes[i, h, j * b: r0] = e4m3_round(old * 2.0 ** (held - e))
                        e = max(e, held)
                    most = 240.0 if e == 120 else 448.0  # 256 * 2^120 is past bf16's end
                    self.codes[i, h, r0:r1] = e4m3_round(new * 2.0 ** -e).clamp(-most, most)
                    self.scale[i, h, j] = e + 127

    def values(self):
        j = torch.arange(self.cap) // self.block
        return self.codes * torch.exp2(self.scale.double() - 127)[:, :, j, None]


def rounded(x, dtype=torch.bfloat16):
    return x.to(torch.float32).to(dtype)


def close(got, want, tol, what):
    """Every element within its own bound (and non-finite ones alike)."""
    got, want = got.double().cpu(), want.double()
    fin = want.isfinite()
    assert torch.equal(got.isfinite(), fin), f"{what}: finite in different places"
    assert torch.equal(got[~fin & ~want.isnan()], want[~fin & ~want.isnan()]), f"{what}: infinities differ"
    if not fin.any():
        return
    over = ((got - want).abs() / tol)[fin]
    i = int(over.argmax())
    assert float(over[i]) <= 1.0, (f"{what}: error {float((got - want).abs()[fin][i]):.3e} of {float(want[fin][i]):.3e} is "
                                   f"{float(over[i]):.2f} times its bound")
