"""The paged 4-bit cache on the GPU: codes, scales and reads bit for bit, attention over it
against float64 on the values that the codes stand for."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests import paged_ref as P
from tests.helpers import lists_to_device

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def pool(S, g, n_pages, H, D, block):
    """A cache of random contents."""
    c = S.PagedCache.empty(n_pages, H, D, block)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        scale.copy_(torch.randint(122, 128, scale.shape, generator=g, dtype=torch.uint8))
    return c


def own_pages(g, B, n, n_pages):
    """Pages [B, n] of the sequences, none of them twice, in random order."""
    return torch.randperm(n_pages, generator=g)[: B * n].view(B, n).int()


def twins(c):
    return [[t.cpu().long() for t in pair] for pair in ((c.k, c.k_scale), (c.v, c.v_scale))]


def same(c, ref, what):
    for (codes, scale), (rc, rs), n in zip(((c.k, c.k_scale), (c.v, c.v_scale)), ref, "kv"):
        assert torch.equal(scale.cpu().long(), rs), f"{what}: {n} scales"
        ok = rc >= 0
        assert torch.equal(codes.cpu().long()[ok], rc[ok]), f"{what}: {n} codes"


def tokens(g, B, H, L, D, packed=False, spread=3.0):
    shape = (B, L, 3, H, D) if packed else (B, H, L, D)
    x = (torch.randn(shape, generator=g) * torch.exp2(spread * torch.randn(*shape[:-1], 1, generator=g))).bfloat16().cuda()
    return [x[:, :, i].transpose(1, 2) for i in (1, 2)] if packed else [x, x.flip(2).contiguous()]


WRITES = [
    # D, block, B, H, L, start, packed, pairs (0: no rotation), interleaved
    (64, 64, 1, 1, 1, 0, False, 0, False),
    (128, 64, 2, 3, 1, 63, True, 64, False),
    (128, 128, 1, 2, 300, 5, False, 64, True),
    (64, 128, 2, 2, 130, 127, True, 24, False),
    (64, 64, 3, 1, 65, 200, False, 8, False),
    (128, 64, 1, 24, 200, 100, True, 40, False),
    (64, 64, 2, 2, 64, 64, False, 16, True),
]


@pytest.mark.parametrize("case", WRITES, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}x{c[4]}-p{c[7]}")
def test_writes(gpu_lib, case):
    D, block, B, H, L, start, packed, pairs, inter = case
    _say(f"[paged write] {case}")
    g = torch.Generator().manual_seed(L + start)
    n = -(-(start + L) // block)
    c = pool(gpu_lib, g, B * n + 3, H, D, block)
    pages, ref = own_pages(g, B, n, B * n + 3), twins(c)
    k, v = tokens(g, B, H, L, D, packed)
    table = P.random_table(g, start + L, pairs) if pairs else None
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), start, table=table.cuda() if pairs else None, interleaved=inter)
    turned = P.turn(k.cpu(), table[start: start + L], pairs, inter) if pairs else k.cpu()
    for x, r in zip((turned, v.cpu()), ref):
        P.write(*r, x, pages, [start] * B)
    torch.cuda.synchronize()
    same(c, ref, "write")
    if pairs:  # the same bits as a rotation first, at positions of its own
        pos = torch.randint(0, start + L, (B, L), generator=g).int().cuda()
        gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), start, table=table.cuda(), positions=pos, interleaved=inter)
        first = [t.clone() for t in c]
        rot = gpu_lib.sparstar_rope_fwd(k, table.cuda(), positions=pos, interleaved=inter)
        gpu_lib.sparstar_paged_write(rot, v, c, pages.cuda(), start)
        assert all(torch.equal(a, b) for a, b in zip(first, c))


def test_padded_batches_and_rows_that_do_not_exist(gpu_lib):
    """Sequences at rows and with counts of their own; rows outside the table and pages outside
    the pool are dropped, shared and foreign pages stay as they were."""
    D, block, B, H, L, n = 64, 64, 6, 2, 70, 4
    g = torch.Generator().manual_seed(4)
    c = pool(gpu_lib, g, B * n + 3, H, D, block)
    pages = own_pages(g, B, n, B * n + 3)
    pages[4, 1], pages[5, 0], pages[5, 1] = -1, B * n + 3, 2 ** 31 - 1
    ref = twins(c)
    k, v = tokens(g, B, H, L, D)
    table = P.random_table(g, n * block, 32)
    starts, counts = [0, 63, 250, -5, 60, 100], [70, 1, 70, 40, 70, 1000]
    dev = dict(dtype=torch.int32, device="cuda")
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), starts=torch.tensor(starts, **dev),
                                 counts=torch.tensor(counts, **dev), table=table.cuda())
    rows = (torch.tensor(starts)[:, None] + torch.arange(L)).clamp(0, n * block - 1)
    for x, r in zip((P.turn(k.cpu(), table[rows][:, None], 32), v.cpu()), ref):
        P.write(*r, x, pages, starts, counts)
    torch.cuda.synchronize()
    same(c, ref, "padded batch")
    counts = [0, -3, 1000, 2, 5, 0]
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda(), 100, counts=torch.tensor(counts, **dev))
    for x, r in zip((k.cpu(), v.cpu()), ref):
        P.write(*r, x, pages, [100] * B, counts)
    torch.cuda.synchronize()
    same(c, ref, "counts alone")
    gpu_lib.sparstar_paged_write(k[:, :, :0], v[:, :, :0], c, pages.cuda(), 256)
    torch.cuda.synchronize()
    same(c, ref, "no tokens")


def test_write_of_unusual_values(gpu_lib):
    """Zeros of both signs, values below bf16's normal range, the largest ones, infinities and
    NaN; largest values just below and above the top of a binade's codes; ties."""
    D, block = 64, 64
    g = torch.Generator().manual_seed(2)
    rows = [torch.full((D,), x) for x in (0.0, -0.0, 1e-40, -1e-39, 3.3e38, -3.38e38, 6.0, 6.03125, 2.0 ** -126, math.inf,
                                          -math.inf, math.nan)]
    odd = torch.randn(6, D, generator=g)
    odd[0, 5], odd[1, 40], odd[2, 2], odd[2, 60], odd[3, 9] = math.inf, -math.inf, math.nan, math.inf, math.nan
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]).repeat(8)
    rows += list(odd) + [ties, -ties, ties * 2.0 ** 30, ties * 2.0 ** -120]
    near = ties.bfloat16().view(torch.int16)
    rows += [(near + 1).view(torch.bfloat16).float().clamp_max(6.0), (near - 1).view(torch.bfloat16).float()]
    x = torch.stack(rows)[None, None].bfloat16()
    c = pool(gpu_lib, g, 1, 1, D, block)
    pages, ref = torch.zeros(1, 1, dtype=torch.int32), twins(c)
    gpu_lib.sparstar_paged_write(x.cuda(), x.cuda(), c, pages.cuda())
    for r in ref:
        P.write(*r, x, pages, [0])
    torch.cuda.synchronize()
    same(c, ref, "unusual values")
    k, v = gpu_lib.sparstar_paged_read(c, pages.cuda(), 0, x.shape[2])
    want = P.decode(ref[0][0].clamp_min(0), ref[0][1])[0, 0, : x.shape[2]]
    got = k[0, 0].cpu().double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()], want[~want.isnan()])
    assert not got.isinf().any() and torch.equal(k.isnan(), v.isnan())


@pytest.mark.parametrize("D,block,start,L", [(64, 64, 0, 1), (128, 64, 63, 2), (128, 128, 5, 300), (64, 128, 127, 130)])
def test_read_is_exact(gpu_lib, D, block, start, L):
    g = torch.Generator().manual_seed(L)
    n, B, H = 5, 2, 3
    c = pool(gpu_lib, g, 12, H, D, block)
    pages = own_pages(g, B, n, 12)
    pages[1, 4], pages[1, 1] = pages[0, 0], 12  # a shared page, and one that does not exist
    _say(f"[paged read] D={D} b={block} {start}+{L}")
    want = []
    for codes, scale in twins(c):
        (u, ok), (s, _) = P.sequence(codes, pages, block), P.sequence(scale, pages, block)
        want.append((P.decode(u, s) * ok[:, None, :, None])[:, :, start: start + L])
    got = gpu_lib.sparstar_paged_read(c, pages.cuda(), start, L)
    assert all(torch.equal(x.cpu().double(), w) for x, w in zip(got, want))
    k, v = gpu_lib.sparstar_paged_read(c, pages.cuda(), start, L, want=("v",))
    assert k is None and torch.equal(v.cpu().double(), want[1])
    pad = torch.full((L * B * H * D + 256,), 9.0, dtype=torch.bfloat16, device="cuda")
    out = pad[:-256].view(B, H, L, D)
    gpu_lib.sparstar_paged_read(c, pages.cuda(), start, L, out=(out, None))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().double(), want[0]) and (pad[-256:] == 9).all()


def attend(S, q, c, pages, lists, Lk, scale, lens, **kw):
    sc = 0.0 if scale == 1 / math.sqrt(q.shape[3]) else scale
    if lists is None:
        return S.sparstar_paged_dense_attn_fwd(q, c, pages, Lk, sc, lens=lens, **kw)
    num, idx = lists_to_device(lists, -(-q.shape[2] // c.block_size))
    return S.sparstar_paged_sparse_attn_fwd(q, c, pages, num, idx, Lk, sc, lens=lens, **kw)


def check(o, lse, q, c, pages, lists, lens, scale):
    """Every row against float64, rows of pages outside the pool left out."""
    B, H, Lq, _ = q.shape
    kv = []
    for codes, scale_bytes in twins(c):
        (u, ok), (s, _) = P.sequence(codes, pages, c.block_size), P.sequence(scale_bytes, pages, c.block_size)
        kv.append(P.decode(u, s))
    for b in range(B):
        m = lens[b]
        for h in range(H):
            mask = R.visible(lists[b][h] if lists is not None else None, Lq, kv[0].shape[2], c.block_size)[:, :m]
            mask = mask & ok[b, None, :m]
            k, v = (x[b, h, :m] for x in kv)
            want = R.forward_tol(q[b, h].double().cpu(), k, v, mask, scale)
            R.close(o[b, h], want[0], want[2], f"o[{b},{h}]")
            R.close(lse[b, h], want[1], want[3], f"lse[{b},{h}]")


ATTEND = [
    # D, block, B, H, Lq, Lk, lens, lists, density, scale factor
    (64, 64, 1, 1, 1, 1, [1], None, 0, 1),
    (128, 128, 1, 2, 1, 700, [700], None, 0, 1),
    (128, 64, 3, 2, 1, 1500, [0, 1, 1500], None, 0, 1),
    (64, 64, 2, 2, 1, 1500, [1477, 65], "random", 0.5, 1),
    (64, 128, 2, 3, 1, 3000, [2999, 127], "holes", 0.5, 2),
    (128, 64, 1, 1, 1, 5000, [5000], None, 0, 4),
    (128, 64, 2, 2, 2, 800, [800, 3], None, 0, 1),
    (128, 64, 4, 1, 3, 333, [63, 64, 65, 333], "random", 0.5, 1),
    (64, 64, 1, 2, 5, 700, [699], None, 0, 1),
    (128, 128, 1, 2, 16, 900, [900], None, 0, 1),
    (64, 128, 2, 3, 31, 2000, [1999, 640], None, 0, 1),
    (128, 64, 1, 2, 32, 4000, [4000], "random", 0.3, 1),
    (128, 64, 1, 2, 33, 500, [500], None, 0, 1),
    (128, 64, 2, 1, 64, 900, [900, 100], "random", 0.4, 1),
    (128, 128, 2, 1, 65, 900, [900, 100], "random", 0.6, 1),
    (64, 64, 1, 2, 200, 1030, [1030], "holes", 0.5, 1),
    (64, 128, 1, 1, 300, 700, [555], "full", 0, 1),
    (128, 64, 1, 1, 200, 333, [0], "full", 0, 1),
    (128, 64, 2, 1, 150, 400, [400, 31], None, 0, 4),
    (64, 64, 1, 2, 129, 400, [400], "one", 0, 0.1),
    (128, 128, 1, 1, 257, 1100, [1100], None, 0, 1),
]


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}-{c[4]}x{c[5]}-{c[7]}")
def test_attention_over_the_pages(gpu_lib, case, split):
    D, block, B, H, Lq, Lk, lens, kind, density, factor = case
    _say(f"[paged attn] {case} split={split}")
    g = torch.Generator().manual_seed(Lk + Lq)
    n = -(-Lk // block)
    c = pool(gpu_lib, g, B * n + 2, H, D, block)
    pages = own_pages(g, B, n, B * n + 2)
    if n > 3 and B > 1:
        pages[1, 2], pages[0, 1] = pages[0, 0], B * n + 2  # a shared page, and one that does not exist
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    scale = factor / math.sqrt(D)
    lists = R.random_lists(g, B, H, -(-Lq // block), n, density, kind) if kind else None
    dl = None if set(lens) == {Lk} else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), lists, Lk, scale, dl, split=split)
    check(o, lse, q, c, pages, lists, lens, scale)
    if split:  # the same bits again, in place of the queries, without lse
        q2 = q.cuda()
        o2, none = attend(gpu_lib, q2, c, pages.cuda(), lists, Lk, scale, dl, out=q2, return_lse=False)
        assert none is None and o2 is q2 and torch.equal(o2, o)


@pytest.mark.parametrize("Lq", [1, 2, 20, 40, 200])
@pytest.mark.parametrize("sparse", [False, True])
def test_rows_past_the_length_are_not_read(gpu_lib, Lq, sparse):
    """NaN scales behind each sequence's rows, a length above Lk and one below zero, pages
    outside the pool behind the end."""
    D, block, B, H, Lk, n = 128, 64, 4, 2, 640, 11
    g = torch.Generator().manual_seed(Lq)
    c = pool(gpu_lib, g, B * n, H, D, block)
    pages = own_pages(g, B, n, B * n)
    lens = [639, 130, 5000, -4]
    for b in range(B):
        for r in range(max(0, min(lens[b], Lk)), n * block):
            for t in (c.k_scale, c.v_scale):
                t[int(pages[b, r // block]), :, r % block] = 255
    pages[1, 5] = -7
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    lists = R.random_lists(g, B, H, -(-Lq // block), n, 0.7) if sparse else None
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), lists, Lk, 1 / math.sqrt(D),
                    torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert not o.isnan().any() and not lse.isnan().any()
    check(o, lse, q, c, pages, lists, [639, 130, Lk, 0], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq", [1, 3, 100])
def test_nan_keys_and_values_are_seen(gpu_lib, Lq):
    """A NaN among the attended values makes the rows that see it NaN, and no others."""
    D, block, H, Lk = 64, 64, 3, 500
    g = torch.Generator().manual_seed(3)
    c = pool(gpu_lib, g, 8, H, D, block)
    pages = own_pages(g, 1, 8, 8)
    c.k_scale[int(pages[0, 2]), 0, 7, 0] = 255
    c.v_scale[int(pages[0, 7]), 1, 9, 1] = 255
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda()
    o, lse = attend(gpu_lib, q, c, pages.cuda(), None, Lk, 1 / math.sqrt(D), None)
    assert o[0, 0].isnan().all() and lse[0, 0].isnan().all()
    assert o[0, 1, :, 32:].isnan().all() and not o[0, 1, :, :32].isnan().any() and lse[0, 1].isfinite().all()
    assert not o[0, 2].isnan().any() and lse[0, 2].isfinite().all()


@pytest.mark.parametrize("Lq", [1, 4, 70])
def test_malformed_lists_read_nothing_outside(gpu_lib, Lq):
    """Entries outside the blocks and counts outside the rows; the rows with good lists are
    right."""
    D, block, H, Lk = 128, 64, 2, 700
    g = torch.Generator().manual_seed(6)
    c = pool(gpu_lib, g, 11, H, D, block)
    pages = own_pages(g, 1, 11, 11)
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16()
    n_q = -(-Lq // block)
    num = torch.full((1, H, n_q), 3, dtype=torch.int32)
    idx = torch.tensor([0, 4, 9], dtype=torch.int32).expand(1, H, n_q, 3).clone()
    num[0, 1], idx[0, 1, :, 1] = 2 ** 30, -5
    idx[0, 1, :, 2] = 2 ** 31 - 1
    o, lse = gpu_lib.sparstar_paged_sparse_attn_fwd(q.cuda(), c, pages.cuda(), num.cuda(), idx.cuda(), Lk)
    lists = [[[[0, 4, 9]] * n_q, [[0]] * n_q]]
    check(o, lse, q, c, pages, lists, [Lk], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq", [1, 40])
def test_offsets_past_32_bits(gpu_lib, Lq):
    """A pool of more than 2^32 bytes of codes, the pages at its end."""
    D, block, H, n = 128, 128, 24, 6
    n_pages = (1 << 32) // (H * block * D // 2) + 3000
    c = gpu_lib.PagedCache.empty(n_pages, H, D, block)
    g = torch.Generator().manual_seed(5)
    pages = torch.tensor([[n_pages - 1, 3, n_pages - 2, n_pages // 2, n_pages - 77, 0]], dtype=torch.int32)
    assert (n_pages - 2) * H * block * D // 2 > 2 ** 32
    L = n * block - 9
    k, v = tokens(g, 1, H, L, D, spread=0.5)
    gpu_lib.sparstar_paged_write(k, v, c, pages.cuda())
    near = gpu_lib.PagedCache.empty(n, H, D, block)
    ordered = torch.arange(n, dtype=torch.int32)[None].cuda()
    gpu_lib.sparstar_paged_write(k, v, near, ordered)
    a, b = gpu_lib.sparstar_paged_read(c, pages.cuda(), 0, L), gpu_lib.sparstar_paged_read(near, ordered, 0, L)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda()
    a = gpu_lib.sparstar_paged_dense_attn_fwd(q, c, pages.cuda(), L)
    b = gpu_lib.sparstar_paged_dense_attn_fwd(q, near, ordered, L)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


JOINS = [  # D, block, H, Lq, Lk, list length (0: dense), ranges
    (128, 64, 1, 1, 9000, 0, 35), (64, 128, 2, 7, 9000, 30, 15), (128, 128, 3, 32, 14_000, 0, 55), (64, 64, 2, 17, 9000, 60, 15),
    (64, 64, 85, 1, 5000, 0, 6), (128, 128, 3, 54, 1724, 0, None), (64, 128, 2, 100, 1100, 0, None), (128, 64, 2, 97, 738, 0, None),
    (128, 128, 4, 130, 2500, 13, None),
    (128, 128, 1, 100, 9000, 0, None), (64, 64, 1, 64, 9000, 60, None), (128, 64, 18, 220, 3500, 0, None),
    (64, 64, 3, 300, 9000, 0, None),
]


@pytest.mark.parametrize("D,block,H,Lq,Lk,stride,ranges", JOINS)
def test_ranges_join(gpu_lib, D, block, H, Lq, Lk, stride, ranges):
    got = gpu_lib.load().sparstar_internal_paged_ranges(1, H, Lq, Lk, D, block, stride)
    _say(f"[paged ranges] {(D, block, H, Lq, Lk, stride)}: {got}")
    assert got > 1 and ranges in (None, got)
    g = torch.Generator().manual_seed(Lk + Lq)
    n = -(-Lk // block)
    c = pool(gpu_lib, g, n, H, D, block)
    pages = own_pages(g, 1, n, n)
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16()
    lists = None
    if stride:
        lists = [[[sorted(torch.randperm(n, generator=g)[:stride].tolist()) for _ in range(-(-Lq // block))] for _ in range(H)]]
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), lists, Lk, 1 / math.sqrt(D), None)
    check(o, lse, q, c, pages, lists, [Lk], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq", [5, 20, 60])
def test_a_nan_query_stays_in_its_row(gpu_lib, Lq):
    D, block, H, Lk = 128, 64, 2, 900
    g = torch.Generator().manual_seed(9)
    c = pool(gpu_lib, g, 15, H, D, block)
    pages = own_pages(g, 1, 15, 15)
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16()
    clean = q.clone()
    q[0, 0, 3, 17] = math.nan
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), None, Lk, 1 / math.sqrt(D), None)
    assert o[0, 0, 3].isnan().all() and lse[0, 0, 3].isnan()
    o[0, 0, 3], lse[0, 0, 3] = 0.0, 0.0
    assert not o.isnan().any() and not lse.isnan().any()
    good = torch.arange(Lq) != 3
    check(o[:, :, good], lse[:, :, good], clean[:, :, good], c, pages, None, [Lk], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq", [1, 20])
def test_many_heads(gpu_lib, Lq):
    """More heads than work-groups at once, of short sequences of every length."""
    D, block, B, H, n = 64, 64, 40, 24, 3
    g = torch.Generator().manual_seed(10)
    c = pool(gpu_lib, g, B * n, H, D, block)
    pages = own_pages(g, B, n, B * n)
    lens = [(7 * b) % (n * block + 1) for b in range(B)]
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    o, lse = attend(gpu_lib, q.cuda(), c, pages.cuda(), None, n * block, 1 / math.sqrt(D),
                    torch.tensor(lens, dtype=torch.int32, device="cuda"))
    pick = [0, 1, 9, 28, 39]
    check(o[pick], lse[pick], q[pick], c, pages[pick], None, [lens[b] for b in pick], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq,block", [(1, 64), (7, 128), (64, 64)])
def test_query_heads_that_share_keys(gpu_lib, Lq, block):
    """Four query heads to a head of the cache are rows of one head; with lists where a head's rows
    are whole blocks, or share one list."""
    D, B, G, H, Lk = 128, 2, 4, 3, 500
    g = torch.Generator().manual_seed(Lq)
    n = -(-Lk // block)
    c, pages = pool(gpu_lib, g, B * n, H, D, block), own_pages(g, B, n, B * n)
    q = torch.randn(B, G * H, Lq, D, generator=g).bfloat16()
    grouped = q.view(B, H, G * Lq, D)
    one = [torch.randperm(n, generator=g)[: n // 2].sort().values.tolist() for _ in range(B * H)]
    blocks = -(-G * Lq // block)
    for lists in (None, [[[one[b * H + h]] * blocks for h in range(H)] for b in range(B)]):
        o, lse = attend(gpu_lib, grouped.cuda(), c, pages.cuda(), lists, Lk, 0.1, None)
        check(o, lse, grouped, c, pages, lists, [Lk] * B, 0.1)
        for i in range(G):  # (each query head by itself: the same rows within the same tolerance)
            alone, few = q.view(B, H, G, Lq, D)[:, :, i], lists and [[x[: -(-Lq // block)] for x in y] for y in lists]
            check(o.view(B, H, G, Lq, D)[:, :, i], lse.view(B, H, G, Lq)[:, :, i], alone, c, pages, few, [Lk] * B, 0.1)


@pytest.mark.parametrize("Lq", [1, 5, 130])
def test_a_step_as_it_is_used(gpu_lib, Lq):
    """Rotation out of a fused projection, append, read for the selector, block-sparse attention:
    eager, on a side stream, and replayed from a graph with another length."""
    S, D, block, B, H, past, n = gpu_lib, 128, 64, 2, 3, 1000, 24
    g = torch.Generator().manual_seed(Lq)
    c = pool(S, g, B * n + 1, H, D, block)
    pages = own_pages(g, B, n, B * n + 1).cuda()
    coords = torch.stack([torch.arange(n * block) // 40, torch.arange(n * block) % 40], dim=1).int().cuda()
    freq, axis = S.sparstar_rope_frequencies(64, factor=2.0, length=700), [i // 32 for i in range(64)]
    table = S.sparstar_rope_table(coords, freq, axis)
    k, v = tokens(g, B, H, past, D, spread=0.3)
    S.sparstar_paged_write(k, v, c, pages, table=table)
    qkv = torch.randn(B, Lq, 3, H, D, generator=g).bfloat16().cuda()
    x = [qkv[:, :, i].transpose(1, 2) for i in range(3)]
    starts = torch.tensor([past, past - 130], dtype=torch.int32, device="cuda")
    Lk = past + Lq
    lens, q = torch.empty_like(starts), torch.empty(B, H, Lq, D, dtype=torch.bfloat16, device="cuda")
    stride = S.sparstar_kv_stride(H, Lk, block, 0.3, [(0, 100)])
    n_q = -(-Lq // block)
    num = torch.empty(B, H, n_q, dtype=torch.int32, device="cuda")
    idx = torch.zeros(B, H, n_q, stride, dtype=torch.int32, device="cuda")
    keys = torch.empty(B, H, Lk, D, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
    scores = torch.empty(S.sparstar_score_workspace_bytes(B, H, Lq, Lk, D, block), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(1, S.sparstar_paged_attn_workspace_bytes(B, H, Lq, Lk, D, block)), dtype=torch.uint8, device="cuda")
    step = torch.arange(Lq, dtype=torch.int32, device="cuda")

    def run():
        at = (starts[:, None] + step).contiguous()
        torch.add(starts, Lq, out=lens)
        S.sparstar_rope_fwd(x[0], table, positions=at, out=q)
        S.sparstar_paged_write(x[1], x[2], c, pages, starts=starts, table=table)
        S.sparstar_paged_read(c, pages, 0, Lk, want=("k",), out=(keys, None))
        S.sparstar_score_blocks(q, keys, block, 0.3, [(0, 100)], kv_stride=stride, out=(num, idx), workspace=scores)
        S.sparstar_paged_sparse_attn_fwd(q, c, pages, num, idx, Lk, lens=lens, out=o, lse=lse, workspace=ws)

    def right():
        torch.cuda.synchronize()
        at = starts.cpu()[:, None].long() + torch.arange(Lq)
        assert torch.equal(q.cpu(), P.turn(x[0].cpu(), table.cpu()[at][:, None], 64))
        lists = [[[idx[b, h, i, : num[b, h, i]].tolist() for i in range(n_q)] for h in range(H)] for b in range(B)]
        check(o, lse, q, c, pages.cpu(), lists, lens.tolist(), 1 / math.sqrt(D))
        new = P.encode(P.turn(x[1].cpu(), table.cpu()[at][:, None], 64))
        for b in range(B):
            rows, _ = P.sequence(c.k.cpu().long(), pages.cpu(), block)
            assert torch.equal(rows[b, :, at[b]], new[0][b])

    run()
    right()
    eager = [t.clone() for t in (q, o, lse, num)]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            run()
    torch.cuda.synchronize()
    for n, shift in enumerate((0, -1, -200, 0)):
        starts.copy_(torch.tensor([past + shift, past - 130], dtype=torch.int32))
        for t in (q, o, keys):
            t.zero_()
        torch.randn(1 << 18, device="cuda").sum().item()
        graph.replay()
        if n == 0:  # (later the rows that the other steps wrote are others)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, (q, o, lse, num)))
        right()
