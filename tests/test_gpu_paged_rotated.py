"""Block-sparse calls over the pages that are large enough for their lists to be walked from a start
that turns with the work-group: which blocks every row sees, and sampled rows against float64."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests import paged_ref as P

pytestmark = pytest.mark.gpu

SHAPES = [  # D, block, B, H, Lq, Lk, list length, lengths of the sequences
    (128, 64, 2, 4, 4000, 84_032, 328, [84_032, 70_001]),
    (64, 64, 2, 4, 11_520, 84_032, 328, [84_031, 60_417]),
    (128, 128, 3, 8, 2000, 84_032, 164, [84_032, 67_226, 50_300]),
    (64, 128, 3, 8, 4000, 84_032, 164, [83_000, 84_032, 40_005]),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"D{s[0]}b{s[1]}-{s[2]}x{s[3]}x{s[4]}")
def test_lists_walked_from_a_turned_start(gpu_lib, shape):
    S, (D, block, B, H, Lq, Lk, stride, lens) = gpu_lib, shape
    i64, out = ctypes.c_int64, (ctypes.c_int64 * 3)()
    S.load().sparstar_internal_paged_plan(B, H, i64(Lq), i64(Lk), D, block, i64(stride), out)
    print(f"[paged rotated] {shape}: waves, ranges, rotation {list(out)}", flush=True)
    assert out[1] > 1 and out[2] > 0
    g = torch.Generator(device="cuda").manual_seed(Lq)
    n_k, n_q = -(-Lk // block), -(-Lq // block)
    n_pages = B * n_k + 1
    c = S.PagedCache.empty(n_pages, H, D, block)
    pages = torch.randperm(n_pages, generator=g, device="cuda")[: B * n_k].view(B, n_k).int()
    pages[1, 5], pages[0, 7], pages[1, 300] = pages[0, 3], -1, n_pages  # one shared, two that do not exist
    idx = torch.rand(B, H, n_q, n_k, generator=g, device="cuda").topk(stride, dim=3).indices.sort(dim=3).values.int().contiguous()
    num = torch.randint(1, stride + 1, (B, H, n_q), generator=g, device="cuda").int()
    num[:, :, 3::5], num[0, 1, 2] = stride, 0
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")

    # 1. Every key weighs the same, and block j has a one in channel j mod D: O counts the listed
    # rows by channel.  Off by O's rounding and by fp32 (whole numbers below 2^24, one quotient).
    # (a page has several tables' blocks: V by page, so the shared page counts for its own)
    exists = (pages >= 0) & (pages < n_pages)
    where = torch.zeros(n_pages, dtype=torch.long, device="cuda")
    order = torch.arange(n_k, device="cuda")
    for b in reversed(range(B)):
        where[pages[b][exists[b]].long()] = order[exists[b]] % D
    c.k.zero_(), c.v.zero_()
    for t in (c.k_scale, c.v_scale):
        t.fill_(127)
    page = torch.arange(n_pages, device="cuda")
    c.v[page, :, :, where // 2] = torch.where(where % 2 == 0, 0x02, 0x20).to(torch.uint8)[:, None, None]
    q = torch.randn(B, H, Lq, D, generator=g, device="cuda").bfloat16()
    o, lse = S.sparstar_paged_sparse_attn_fwd(q, c, pages, num, idx, Lk, lens=lt)
    rows = (lt[:, None].long() - order * block).clamp(0, block) * exists  # of each block, [B, n_k]
    channel = where[pages.clamp(0, n_pages - 1).long()]  # [B, n_k]
    listed = torch.arange(stride, device="cuda") < num[..., None]
    at = idx.long()
    b_of = torch.arange(B, device="cuda")[:, None, None, None].expand_as(at)
    w = (rows[b_of, at] * listed).double()
    want = torch.zeros(B, H, n_q, D, dtype=torch.float64, device="cuda").scatter_add_(3, channel[b_of, at], w)
    total = w.sum(dim=3)
    block_of = torch.arange(Lq, device="cuda") // block
    want = (want / total.clamp_min(1)[..., None])[:, :, block_of]
    assert ((o.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want).all()
    lw = total.log()[:, :, block_of]
    assert torch.equal(lse.isinf(), lw.isinf()) and (lse[~lse.isinf()] - lw[~lw.isinf()]).abs().max() < 2.0 ** -18

    # 2. random contents
    for t in (c.k, c.v):
        t.random_(0, 256, generator=g)
    for t in (c.k_scale, c.v_scale):
        t.random_(122, 128, generator=g)
    o, lse = S.sparstar_paged_sparse_attn_fwd(q, c, pages, num, idx, Lk, lens=lt)
    codes = [t.cpu() for t in c]
    pg, ix, nm = pages.cpu().long(), idx.cpu().long(), num.cpu()
    for b in range(B):
        for h in (0, 1, H - 1):
            for i in (0, 2, n_q // 2, n_q - 9, n_q - 1):
                mine = ix[b, h, i, : nm[b, h, i]]
                mine = mine[exists[b].cpu()[mine]]
                p = pg[b, mine]
                k, v = (P.decode(codes[n][p, h], codes[n + 2][p, h]).flatten(0, 1) for n in (0, 1))
                mask = ((mine[:, None] * block + torch.arange(block)) < lens[b]).flatten()
                r = slice(i * block, min(Lq, (i + 1) * block))
                x = q[b, h, r].double().cpu()
                ref = R.forward_tol(x, k, v, mask[None].expand(x.shape[0], -1), 1 / math.sqrt(D))
                R.close(o[b, h, r], ref[0], ref[2], f"o[{b},{h}] block {i}")
                R.close(lse[b, h, r], ref[1], ref[3], f"lse[{b},{h}] block {i}")
