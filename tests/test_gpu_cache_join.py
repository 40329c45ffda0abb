"""Attention over the 8-bit cache where a list is cut into parts: every part of the join can be
seen in the result.  Each part's values have a column of their own, so that O's column says what
that part added, whatever the others hold."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device
from tests.test_gpu_cache import values_of
from tests.test_ops_abi import cache_plan

pytestmark = pytest.mark.gpu

CASES = [
    # D, block, H, Lq, cap, listed blocks (0: dense)
    (128, 64, 1, 1, 9000, 0),
    (128, 64, 1, 3, 16_000, 120),
    (64, 128, 2, 1, 9001, 0),
    (64, 64, 1, 32, 9000, 60),
    (128, 128, 1, 100, 9000, 0),
    (64, 64, 1, 64, 30_000, 100),
]


def inputs(case, parts):
    """q, k, v [1, H, L, D], each head's list of blocks, and each token's part (-1: not listed).
    A part holds its even share of the list's entries."""
    D, block, H, Lq, cap, stride = case
    g = torch.Generator().manual_seed(cap + Lq)
    q, k = torch.randn(1, H, Lq, D, generator=g), torch.randn(1, H, cap, D, generator=g)
    v = torch.randn(1, H, cap, D, generator=g)
    lists, part_of = [], torch.full((H, cap), -1)
    for h in range(H):
        n_k = -(-cap // block)
        lists.append(sorted(torch.randperm(n_k, generator=g)[:stride].tolist()) if stride else list(range(n_k)))
        n = len(lists[h])
        for p in range(parts):
            for j in lists[h][n * p // parts: n * (p + 1) // parts]:
                part_of[h, j * block:(j + 1) * block] = p
        own = part_of[h][:, None] == torch.arange(parts)
        v[0, h, :, :parts] = own * (2 + torch.rand(cap, 1, generator=g))
    return q.bfloat16(), k.bfloat16(), v.bfloat16(), lists, part_of


def seen(q, k, v, lists, part_of, parts, block, scale):
    """(o, lse and their bounds) of one head, after making sure that no part could be missing,
    or weigh 4% more or less, without O leaving its bound."""
    Lq, cap = q.shape[0], k.shape[0]
    mask = R.visible([lists] * -(-Lq // block), Lq, cap, block)
    want = R.forward_tol(q, k, v, mask, scale)
    p = R.forward(q, k, v, mask, scale)[2]
    for i in range(parts):
        mine = (part_of == i).double()
        added = (p * mine) @ v[:, i]
        assert (0.04 * added > 2 * want[2][:, i]).all(), i
    return want


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}-{c[3]}x{c[4]}-{c[5]}")
def test_every_part_is_joined(gpu_lib, case):
    S = gpu_lib
    D, block, H, Lq, cap, stride = case
    parts = cache_plan(S.load(), 1, H, Lq, cap, D, block, stride)[1]
    print(f"[cache join] {case}: {parts} parts", flush=True)
    assert 1 < parts <= D
    q, k, v, lists, part_of = inputs(case, parts)
    c = S.KvCache.empty(1, H, cap, D, block)
    S.sparstar_cache_write(k.cuda(), v.cuda(), c)
    if stride:
        num, idx = lists_to_device([[[l] * -(-Lq // block) for l in lists]], -(-Lq // block))
        o, lse = S.sparstar_cache_sparse_attn_fwd(q.cuda(), c, num, idx)
    else:
        o, lse = S.sparstar_cache_dense_attn_fwd(q.cuda(), c)
    kv = values_of(c)
    for h in range(H):
        x = [q[0, h].double(), kv[0][0, h], kv[1][0, h]]
        want = seen(*x, lists[h], part_of[h], parts, block, 1 / math.sqrt(D))
        R.close(o[0, h], want[0], want[2], f"o[{h}]")
        R.close(lse[0, h], want[1], want[3], f"lse[{h}]")


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}-{c[3]}x{c[4]}-{c[5]}")
def test_what_the_join_rounds(gpu_lib, case, split):
    """All logits are zero, so that P is 1 and nothing is rounded but the ranges' sums A_r (to
    fp16, by 2^-11, in a call that is cut) and O (to bf16, by 2^-8).  fp32 sums of up to 30,000
    terms: 2^-24 of Sum |v| per addition, some 30 of them in a row per sub-tile and as many
    levels above, far below 2^-16 of it.  Columns differ by up to 2^12 in size."""
    S = gpu_lib
    D, block, H, Lq, cap, stride = case
    parts = cache_plan(S.load(), 1, H, Lq, cap, D, block, stride)[1]
    _, k, v, lists, part_of = inputs(case, parts)
    v = (v.float() * torch.exp2(-(torch.arange(D) % 13).float())).bfloat16()
    c = S.KvCache.empty(1, H, cap, D, block)
    S.sparstar_cache_write(k.cuda(), v.cuda(), c)
    q = torch.zeros(1, H, Lq, D, dtype=torch.bfloat16)
    if stride:
        num, idx = lists_to_device([[[l] * -(-Lq // block) for l in lists]], -(-Lq // block))
        o, lse = S.sparstar_cache_sparse_attn_fwd(q.cuda(), c, num, idx, split=split)
    else:
        o, lse = S.sparstar_cache_dense_attn_fwd(q.cuda(), c, split=split)
    for h in range(H):
        vd = values_of(c)[1][0, h]
        n = int((part_of[h] >= 0).sum())
        sums = torch.stack([vd[part_of[h] == p].sum(dim=0) for p in range(parts)])
        want, size = sums.sum(dim=0) / n, vd[part_of[h] >= 0].abs().sum(dim=0) / n
        kept = sums.abs().sum(dim=0) / n * 2.0 ** -11 + parts * float(sums.abs().max()) / n * 2.0 ** -39 if split else 0
        inner = kept + 2.0 ** -16 * size
        tol = (R.U * (want.abs() + inner) + inner).expand(Lq, D)
        R.close(o[0, h], want.expand(Lq, D), tol, f"o[{h}]")
        R.close(lse[0, h], torch.full((Lq,), math.log(n), dtype=torch.float64),
                torch.full((Lq,), 2.0 ** -20 * (1 + math.log(n)), dtype=torch.float64), f"lse[{h}]")
