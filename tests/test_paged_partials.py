"""What the ranges of a call over the paged cache leave for their join: sums in fp32, whatever the
magnitudes of the other channels, in a workspace that holds them."""
from __future__ import annotations

import math
import random

import pytest
import torch

from paper_2608_10519_amd import sparstar as S
from tests import grad_cache_ref as R
from tests import paged_ref as P
from tests.test_gpu_paged import attend, check, own_pages, pool, twins


def test_the_workspace_holds_the_sums():
    """D sums, two row sums and a maximum of every range and row, in 32 bits."""
    rng = random.Random(3)
    cut = 0
    for _ in range(400):
        B, H, D, block = rng.randint(1, 3), rng.randint(1, 30), rng.choice([64, 128]), rng.choice([64, 128])
        Lq, Lk = round(math.exp(rng.uniform(0, 9))), round(math.exp(rng.uniform(3, 12)))
        stride = rng.choice([0, rng.randint(1, -(-Lk // block))])
        ranges = S.load().sparstar_internal_paged_ranges(B, H, Lq, Lk, D, block, stride)
        size = S.sparstar_paged_attn_workspace_bytes(B, H, Lq, Lk, D, block)
        assert size >= (ranges > 1) * ranges * B * H * Lq * 4 * (D + 3)
        cut += ranges > 1
    assert cut > 100


CUT = [  # D, block, H, Lq, Lk, list length (0: dense)
    (128, 64, 1, 7, 9000, 0), (128, 128, 3, 54, 1724, 0), (64, 128, 2, 100, 1100, 0), (64, 64, 1, 64, 9000, 60),
    (128, 128, 4, 130, 2500, 13), (128, 64, 18, 220, 3500, 0), (128, 64, 2, 400, 9000, 100),
]


def _cut(S, g, D, block, H, Lq, Lk, stride):
    assert S.load().sparstar_internal_paged_ranges(1, H, Lq, Lk, D, block, stride) > 1
    n = -(-Lk // block)
    c, pages = pool(S, g, n, H, D, block), own_pages(g, 1, n, n)
    lists = None
    if stride:
        lists = [[[sorted(torch.randperm(n, generator=g)[:stride].tolist()) for _ in range(-(-Lq // block))] for _ in range(H)]]
    return c, pages, lists, torch.randn(1, H, Lq, D, generator=g).bfloat16()


@pytest.mark.gpu
@pytest.mark.parametrize("case", CUT, ids=str)
def test_channels_of_very_different_magnitude(gpu_lib, case):
    """Groups of 32 channels 2^40 and more apart: each column within the roundings of its own
    values (P's and O's to bf16)."""
    print(f"[paged partials] {case}", flush=True)
    D, Lk = case[0], case[4]
    g = torch.Generator().manual_seed(Lk)
    c, pages, lists, q = _cut(gpu_lib, g, *case)
    for i, e in enumerate((60, -60) if D == 64 else (-20, 60, -60, 20)):
        c.v_scale[..., i] = 127 + e
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), lists, Lk, 1 / math.sqrt(D), None)
    check(o, lse, q, c, pages, lists, [Lk], 1 / math.sqrt(D))


@pytest.mark.gpu
@pytest.mark.parametrize("case", CUT, ids=str)
def test_sums_past_the_largest_number_stay_in_their_channels(gpu_lib, case):
    """Values at the end of the range, whose sum is infinite in 32 channels; the others are right."""
    print(f"[paged partials] {case}", flush=True)
    D, block, H, Lq, Lk, _ = case
    g = torch.Generator().manual_seed(Lk + 1)
    c, pages, lists, q = _cut(gpu_lib, g, *case)
    c.v[..., :16], c.v_scale[..., 0] = 0x77, 127 + 125  # 6 * 2^125 throughout
    c.v_scale[..., 1] = 127 - 30
    if D == 128:
        c.v_scale[..., 2] = 127 + 20
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), lists, Lk, 1 / math.sqrt(D), None)
    (k, ks), (v, vs) = twins(c)
    k, v = (P.decode(P.sequence(a, pages, block)[0], P.sequence(b, pages, block)[0])[0, :, :Lk] for a, b in ((k, ks), (v, vs)))
    assert not o[..., :32].isfinite().any()
    for h in range(H):
        mask = R.visible(lists[0][h] if lists else None, Lq, -(-Lk // block) * block, block)[:, :Lk]
        want = R.forward_tol(q[0, h].double(), k[h], v[h, :, 32:], mask, 1 / math.sqrt(D))
        R.close(o[0, h, :, 32:], want[0], want[2], f"o[{h}]")
        R.close(lse[0, h], want[1], want[3], f"lse[{h}]")
