"""The paged cache's writes of many rows, four heads to a thread, and its reads of many bytes, two
chunks to a thread: codes, scales and values bit for bit against the definition."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_ref as P
from tests.test_gpu_paged import own_pages, pool, same, tokens, twins

pytestmark = pytest.mark.gpu

FOUR_HEADS = 8192  # rows of all sequences and heads from which a thread of a write takes four heads


def _say(msg):
    print(msg, flush=True)


def spoiled(g, x):
    """Some groups of 32 channels with infinities, NaN, zeros and the ends of the range in them."""
    for value in (math.inf, -math.inf, math.nan, 3.38e38, 1e-40, 0.0):
        at = torch.randint(0, x[..., 0].numel(), (40,), generator=g)
        x.view(-1, x.shape[-1])[at, torch.randint(0, x.shape[-1], (40,), generator=g)] = value
    x.view(-1, x.shape[-1])[torch.randint(0, x[..., 0].numel(), (9,), generator=g)] = 0.0


WRITES = [
    # D, block, B, H, L, start, packed, pairs (0: no rotation), interleaved
    (128, 64, 2, 5, 900, 100, True, 64, False),
    (64, 128, 1, 6, 1500, 5, True, 24, False),
    (64, 64, 1, 7, 1171, 63, False, 16, True),
    (128, 128, 3, 4, 700, 0, False, 40, True),
    (128, 64, 1, 24, 400, 77, True, 0, False),
    (64, 64, 1, 1, 8209, 1, False, 32, False),
    (128, 128, 4, 9, 333, 130, False, 8, False),
    (64, 64, 3, 2731, 1, 70, False, 32, True),
]


@pytest.mark.parametrize("case", WRITES, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}x{c[4]}-p{c[7]}")
def test_writes_of_four_heads_a_thread(gpu_lib, case):
    D, block, B, H, L, start, packed, pairs, inter = case
    _say(f"[paged write] {case}")
    assert B * H * L >= FOUR_HEADS
    g = torch.Generator().manual_seed(L + start)
    n = -(-(start + L) // block)
    c = pool(gpu_lib, g, B * n + 3, H, D, block)
    pages, ref = own_pages(g, B, n, B * n + 3), twins(c)
    k, v = tokens(g, B, H, L, D, packed)
    if not packed:
        for t in (k, v):
            host = t.cpu()
            spoiled(g, host)
            t.copy_(host)
    table = P.random_table(g, start + L, pairs) if pairs else None
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), start, table=table.cuda() if pairs else None, interleaved=inter)
    turned = P.turn(k.cpu(), table[start: start + L], pairs, inter) if pairs else k.cpu()
    for x, r in zip((turned, v.cpu()), ref):
        P.write(*r, x, pages, [start] * B)
    torch.cuda.synchronize()
    same(c, ref, "write")


@pytest.mark.parametrize("D,block,H,pairs,inter", [(64, 64, 5, 32, False), (128, 128, 3, 24, True), (128, 64, 6, 0, False)])
def test_padded_batches_of_four_heads_a_thread(gpu_lib, D, block, H, pairs, inter):
    """Rows and counts of each sequence, tokens outside the table's rows, pages outside the pool."""
    B, L = 6, 500
    assert B * H * L >= FOUR_HEADS
    g = torch.Generator().manual_seed(H)
    n = -(-700 // block)
    c = pool(gpu_lib, g, B * n + 3, H, D, block)
    pages = own_pages(g, B, n, B * n + 3)
    pages[4, 1], pages[5, 0], pages[5, 1] = -1, B * n + 3, 2 ** 31 - 1
    ref = twins(c)
    k, v = tokens(g, B, H, L, D)
    table = P.random_table(g, n * block, pairs) if pairs else None
    starts, counts = [0, 63, 400, -5, 60, 100], [500, 1, 500, 499, 500, 1000]
    dev = dict(dtype=torch.int32, device="cuda")
    pos = torch.randint(0, n * block, (B, L), generator=g)
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), starts=torch.tensor(starts, **dev),
                                 counts=torch.tensor(counts, **dev), table=table.cuda() if pairs else None,
                                 positions=pos.int().cuda() if pairs else None, interleaved=inter)
    turned = P.turn(k.cpu(), table[pos][:, None], pairs, inter) if pairs else k.cpu()
    for x, r in zip((turned, v.cpu()), ref):
        P.write(*r, x, pages, starts, counts)
    torch.cuda.synchronize()
    same(c, ref, "padded batch")


@pytest.mark.parametrize("D,H,L,want", [(128, 3, 126_001, "kv"), (128, 7, 107_159, "k"), (64, 5, 150_007, "kv"),
                                        (64, 11, 136_391, "v")])
def test_reads_of_many_bytes(gpu_lib, D, H, L, want):
    """More than 192 MB, from inside a page to inside a page, with pages that do not exist: the same
    rows as reads of a few pages."""
    assert 2 * D * H * L * len(want) > 192e6
    _say(f"[paged read] {want}, D={D}, {H} heads of {L} rows")
    block, start, n = 64, 37, 90
    g = torch.Generator().manual_seed(L)
    c = pool(gpu_lib, g, n, H, D, block)
    pages = torch.randint(-1, n + 1, (1, -(-(start + L) // block)), generator=g)
    each = torch.arange(n, dtype=torch.int32)[:, None]
    rows = gpu_lib.sparstar_paged_read(c, each.cuda(), 0, block)  # [n, H, block, D]
    for codes, r in zip(twins(c), rows):  # (and those as the definition has them)
        assert torch.equal(r.cpu().double(), P.decode(*codes))
    got = gpu_lib.sparstar_paged_read(c, pages.int().cuda(), start, L, want=tuple(want))
    for name, x, r in zip("kv", got, rows):
        if name not in want:
            assert x is None
            continue
        exists = ((pages >= 0) & (pages < n)).cuda()[0]
        whole = r[pages.clamp(0, n - 1).cuda()[0]] * exists[:, None, None, None]  # [pages, H, block, D]
        assert torch.equal(x[0], whole.transpose(0, 1).flatten(1, 2)[:, start: start + L])
