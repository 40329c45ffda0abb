"""GPU parity of the 8-bit cache: codes and scales are what the definition gives, bit for
bit; attention over it against float64 on the values that the codes stand for."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device
from tests.test_ops_abi import cache_plan

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def values_of(cache):
    """(k, v) of a whole cache as float64 on the CPU, by the definition."""
    out = []
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        j = torch.arange(codes.shape[2]) // cache.block_size
        out.append(codes.cpu().float().double() * torch.exp2(scale.cpu().double() - 127)[:, :, j, None])
    return out


def blank(S, B, H, cap, D, block, seed=1):
    """A cache of random (valid) contents and its float64 twin."""
    c = S.KvCache.empty(B, H, cap, D, block)
    g = torch.Generator().manual_seed(seed)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        raw = torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8)
        raw[(raw & 0x7f) == 0x7f] = 5  # no NaN
        codes.view(torch.uint8).copy_(raw)
        scale.copy_(torch.randint(118, 125, scale.shape, generator=g, dtype=torch.uint8))
    return c


def twins(c):
    B, H, cap, D = c.k.shape
    return [R.RefCache(B, H, cap, D, c.block_size, codes.cpu().float().double(), scale.cpu().long())
            for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale))]


def same(c, ref, what):
    for codes, scale, r, n in ((c.k, c.k_scale, ref[0], "k"), (c.v, c.v_scale, ref[1], "v")):
        assert torch.equal(scale.cpu().long(), r.scale), f"{what}: {n} scales"
        got = codes.cpu().float().double()
        assert torch.equal(got.isnan(), r.codes.isnan()), f"{what}: {n} NaN"
        ok = ~got.isnan()
        assert torch.equal(got[ok], r.codes[ok]), f"{what}: {n} codes"


def tokens(g, B, H, L, D, spread=3.0):
    x = torch.randn(B, H, L, D, generator=g)
    return (x * torch.exp2(spread * torch.randn(B, H, L, 1, generator=g))).bfloat16()


@pytest.mark.parametrize("D,block", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_writes_in_a_row(gpu_lib, D, block):
    """Chunks of odd lengths one after the other: whole blocks, single tokens, a block
    continued by larger and by smaller values."""
    B, H, cap = 2, 2, 5 * block + 13
    c = blank(gpu_lib, B, H, cap, D, block)
    ref = twins(c)
    g = torch.Generator().manual_seed(D + block)
    pos = 0
    for n, L in enumerate((1, 1, block - 2, 3, block + 1, 7, 1, 2 * block, 0, 5)):
        k, v = tokens(g, B, H, L, D), tokens(g, B, H, L, D)
        _say(f"[cache write] D={D} b={block} rows {pos}..{pos + L}")
        gpu_lib.sparstar_cache_write(k.cuda(), v.cuda(), c, pos)
        for x, r in zip((k, v), ref):
            r.write(x.double(), [pos] * B)
        torch.cuda.synchronize()
        same(c, ref, f"write {n}")
        pos += L
    # to the very end, and over what was there before
    L = cap - pos
    k, v = tokens(g, B, H, L, D), tokens(g, B, H, L, D)
    gpu_lib.sparstar_cache_write(k.cuda(), v.cuda(), c, pos)
    for x, r in zip((k, v), ref):
        r.write(x.double(), [pos] * B)
    k, v = tokens(g, B, H, block + 3, D), tokens(g, B, H, block + 3, D)
    gpu_lib.sparstar_cache_write(k.cuda(), v.cuda(), c, 9)
    for x, r in zip((k, v), ref):
        r.write(x.double(), [9] * B)
    torch.cuda.synchronize()
    same(c, ref, "end")


def test_write_of_unusual_values(gpu_lib):
    """Zeros, values below bf16's normal range, the largest ones, infinities and NaN;
    values whose largest lies just below and above the top of a binade's codes."""
    D, block = 64, 64
    rows = [torch.zeros(block, D), torch.full((block, D), 1e-40), torch.full((block, D), 3.3e38),
            torch.full((block, D), 448.0), torch.full((block, D), 450.0), torch.full((block, D), 2.0 ** -126)]
    g = torch.Generator().manual_seed(2)
    odd = torch.randn(block, D, generator=g)
    odd[3, 5], odd[7, 1], odd[9, 2] = math.inf, -math.inf, math.nan
    rows += [odd, torch.full((block, D), math.nan), torch.full((block, D), math.inf)]
    x = torch.cat(rows)[None, None].bfloat16()
    c = blank(gpu_lib, 1, 1, x.shape[2], D, block)
    ref = twins(c)
    gpu_lib.sparstar_cache_write(x.cuda(), x.cuda(), c)
    for r in ref:
        r.write(x.double(), [0])
    torch.cuda.synchronize()
    same(c, ref, "unusual values")
    k, v = gpu_lib.sparstar_cache_read(c, 0, x.shape[2])
    want = ref[0].values()[0, 0]
    got = k[0, 0].cpu().double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()], want[~want.isnan()])
    assert torch.equal(k.isnan(), v.isnan())


def test_padded_batches(gpu_lib):
    """Every sequence at its own row with its own count; rows outside the cache dropped."""
    D, block, B, H, cap, L = 128, 64, 5, 2, 300, 70
    c = blank(gpu_lib, B, H, cap, D, block, 3)
    ref = twins(c)
    g = torch.Generator().manual_seed(4)
    k, v = tokens(g, B, H, L, D), tokens(g, B, H, L, D)
    starts, counts = [0, 63, 250, -5, 300], [70, 1, 70, 40, 70]
    dev = dict(dtype=torch.int32, device="cuda")
    gpu_lib.sparstar_cache_write(k.cuda(), v.cuda(), c, starts=torch.tensor(starts, **dev),
                                 counts=torch.tensor(counts, **dev))
    for x, r in zip((k, v), ref):
        r.write(x.double(), starts, counts)
    torch.cuda.synchronize()
    same(c, ref, "padded batch")
    counts = [0, -3, 1000, 2, 5]
    gpu_lib.sparstar_cache_write(k.cuda(), v.cuda(), c, 100, counts=torch.tensor(counts, **dev))
    for x, r in zip((k, v), ref):
        r.write(x.double(), [100] * B, counts)
    torch.cuda.synchronize()
    same(c, ref, "counts alone")


@pytest.mark.parametrize("D,block,start,L", [(64, 64, 0, 1), (128, 64, 63, 2), (128, 128, 5, 300), (64, 128, 127, 130)])
def test_read_is_exact(gpu_lib, D, block, start, L):
    c = blank(gpu_lib, 2, 3, 501, D, block, 7)
    _say(f"[cache read] D={D} b={block} {start}+{L}")
    want = values_of(c)
    k, v = gpu_lib.sparstar_cache_read(c, start, L)
    for got, w in zip((k, v), want):
        assert torch.equal(got.cpu().double(), w[:, :, start:start + L])
    k, v = gpu_lib.sparstar_cache_read(c, start, L, want=("v",))
    assert k is None and torch.equal(v.cpu().double(), want[1][:, :, start:start + L])
    pad = torch.full((L * 2 * 3 * D + 256,), 9.0, dtype=torch.bfloat16, device="cuda")
    out = pad[:-256].view(2, 3, L, D)
    gpu_lib.sparstar_cache_read(c, start, L, out=(out, None))
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().double(), want[0][:, :, start:start + L]) and (pad[-256:] == 9).all()


def attend(S, q, c, lists, Lk, scale, lens, **kw):
    D = q.shape[3]
    sc = 0.0 if scale == 1 / math.sqrt(D) else scale
    if lists is None:
        return S.sparstar_cache_dense_attn_fwd(q, c, Lk, sc, lens=lens, **kw)
    num, idx = lists_to_device(lists, -(-q.shape[2] // c.block_size))
    return S.sparstar_cache_sparse_attn_fwd(q, c, num, idx, Lk, sc, lens=lens, **kw)


def check_attention(o, lse, q, c, lists, lens, scale):
    kv = values_of(c)
    B, H, Lq, D = q.shape
    for b in range(B):
        for h in range(H):
            m = lens[b]
            mask = R.visible(lists[b][h] if lists is not None else None, Lq, c.k.shape[2], c.block_size)[:, :m]
            want = R.forward_tol(q[b, h].double(), kv[0][b, h, :m], kv[1][b, h, :m], mask, scale)
            R.close(o[b, h], want[0], want[2], f"o[{b},{h}]")
            R.close(lse[b, h], want[1], want[3], f"lse[{b},{h}]")


def filled(S, g, B, H, cap, D, block, spread=1.0):
    c = S.KvCache.empty(B, H, cap, D, block)
    S.sparstar_cache_write(tokens(g, B, H, cap, D, spread).cuda(), tokens(g, B, H, cap, D, spread).cuda(), c)
    return c


ATTEND = [
    # D, block, B, H, Lq, cap, lens, lists, density, scale factor
    (64, 64, 1, 1, 1, 1, [1], None, 0, 1),
    (128, 128, 1, 2, 1, 700, [700], None, 0, 1),
    (128, 64, 3, 2, 1, 1500, [0, 1, 1500], None, 0, 1),
    (128, 64, 4, 1, 3, 333, [63, 64, 65, 333], "random", 0.5, 1),
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
def test_attention_over_the_cache(gpu_lib, case, split):
    D, block, B, H, Lq, cap, lens, kind, density, factor = case
    _say(f"[cache attn] {case} split={split}")
    g = torch.Generator().manual_seed(cap + Lq)
    c = filled(gpu_lib, g, B, H, cap, D, block)
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    scale = factor / math.sqrt(D)
    lists = R.random_lists(g, B, H, -(-Lq // block), -(-cap // block), density, kind) if kind else None
    dl = None if set(lens) == {cap} else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = attend(gpu_lib, q.cuda(), c, lists, cap, scale, dl, split=split)
    check_attention(o, lse, q, c, lists, lens, scale)


@pytest.mark.parametrize("D,block,H,Lq,cap,stride", [(128, 64, 1, 1, 9000, 0), (64, 128, 2, 7, 9000, 30),
                                                     (128, 128, 1, 100, 9000, 0), (64, 64, 1, 64, 9000, 60)])
def test_ranges_join(gpu_lib, D, block, H, Lq, cap, stride):
    plan = cache_plan(gpu_lib.load(), 1, H, Lq, cap, D, block, stride)
    _say(f"[cache ranges] {(D, block, H, Lq, cap, stride)}: {plan}")
    assert plan[1] > 1
    g = torch.Generator().manual_seed(cap + Lq)
    c = filled(gpu_lib, g, 1, H, cap, D, block)
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16()
    lists = None
    if stride:
        lists = [[[sorted(torch.randperm(-(-cap // block), generator=g)[:stride].tolist())
                   for _ in range(-(-Lq // block))] for _ in range(H)]]
    o, lse = attend(gpu_lib, q.cuda(), c, lists, cap, 1 / math.sqrt(D), None)
    check_attention(o, lse, q, c, lists, [cap], 1 / math.sqrt(D))


@pytest.mark.parametrize("Lq", [1, 40, 200])
@pytest.mark.parametrize("sparse", [False, True])
def test_rows_past_the_length_are_not_read(gpu_lib, Lq, sparse):
    """NaN codes and NaN scales behind each sequence's rows, a length above Lk."""
    D, block, B, H, cap, Lk = 128, 64, 3, 2, 700, 640
    g = torch.Generator().manual_seed(Lq)
    lens, clamped = [77, 0, 9999], [77, 0, Lk]
    c = filled(gpu_lib, g, B, H, cap, D, block)
    for b in range(B):
        for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
            codes.view(torch.uint8)[b, :, clamped[b]:] = 0x7f
            scale[b, :, -(-clamped[b] // block):] = 255
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    lists = R.random_lists(g, B, H, -(-Lq // block), -(-Lk // block), 0.7) if sparse else None
    o, lse = attend(gpu_lib, q.cuda(), c, lists, Lk, 1 / math.sqrt(D), torch.tensor(lens, dtype=torch.int32).cuda())
    check_attention(o, lse, q, c, lists, clamped, 1 / math.sqrt(D))
    assert not o[1].any() and (lse[1] == -math.inf).all()


def test_malformed_lists(gpu_lib):
    D, block, cap = 64, 64, 300
    g = torch.Generator().manual_seed(8)
    c = filled(gpu_lib, g, 1, 1, cap, D, block)
    for Lq in (20, 64):
        q = torch.randn(1, 1, Lq, D, generator=g).bfloat16()
        num = torch.tensor([[[9]]], dtype=torch.int32).cuda()
        idx = torch.tensor([[[[-4, 1, 3, 5, 99]]]], dtype=torch.int32).cuda()
        o, lse = gpu_lib.sparstar_cache_sparse_attn_fwd(q.cuda(), c, num, idx)
        check_attention(o, lse, q, c, [[[[1, 3]]]], [cap], 1 / math.sqrt(D))
        o, lse = gpu_lib.sparstar_cache_sparse_attn_fwd(q.cuda(), c, num * 0 - 2, idx)
        assert not o.any() and (lse == -math.inf).all()


def test_nan_queries_stay_nan(gpu_lib):
    D, block, cap = 128, 64, 3000
    g = torch.Generator().manual_seed(9)
    c = filled(gpu_lib, g, 1, 1, cap, D, block)
    for Lq in (4, 100):
        q = torch.randn(1, 1, Lq, D, generator=g).bfloat16()
        q[0, 0, 2, 7] = math.nan
        o, lse = gpu_lib.sparstar_cache_dense_attn_fwd(q.cuda(), c)
        assert o[0, 0, 2].isnan().all() and bool(lse[0, 0, 2].isnan())
        rest = [i for i in range(Lq) if i != 2]
        assert o[0, 0, rest].isfinite().all() and lse[0, 0, rest].isfinite().all()


def test_shared_heads_as_one_head(gpu_lib):
    """Four query heads over each cache head, one token: the same as four heads that hold
    copies of it."""
    D, block, Hk, G, cap = 128, 64, 2, 4, 1000
    g = torch.Generator().manual_seed(10)
    c = filled(gpu_lib, g, 1, Hk, cap, D, block)
    q = torch.randn(1, Hk * G, 1, D, generator=g).bfloat16()
    o, lse = gpu_lib.sparstar_cache_dense_attn_fwd(q.cuda().view(1, Hk, G, D), c)
    wide = gpu_lib.KvCache(*[t.view(torch.uint8).repeat_interleave(G, dim=1).view(t.dtype) for t in c[:4]], block)
    check_attention(o.view(1, Hk * G, 1, D), lse.view(1, Hk * G, 1), q, wide, None, [cap], 1 / math.sqrt(D))


def test_serving_run(gpu_lib):
    """A clip's step: reference and text written, the scale's own keys appended, blocks
    selected on the keys read back, sparse attention over the cache; the bf16 forward on
    the keys read back agrees with it."""
    S = gpu_lib
    D, block, B, H, Lref, Lq = 128, 64, 2, 2, 500, 330
    Lk = Lref + Lq
    g = torch.Generator().manual_seed(11)
    c = S.KvCache.empty(B, H, 1000, D, block)
    k, v = tokens(g, B, H, Lk, D, 0.5), tokens(g, B, H, Lk, D, 0.5)
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16().cuda()
    S.sparstar_cache_write(k[:, :, :Lref].contiguous().cuda(), v[:, :, :Lref].contiguous().cuda(), c)
    S.sparstar_cache_write(k[:, :, Lref:].contiguous().cuda(), v[:, :, Lref:].contiguous().cuda(), c, Lref)
    kb, vb = S.sparstar_cache_read(c, 0, Lk)
    num, idx = S.sparstar_score_blocks(q, kb, block, 0.5, [(0, 100)])
    o, lse = S.sparstar_cache_sparse_attn_fwd(q, c, num, idx, Lk)
    o2, lse2 = S.sparstar_sparse_attn_fwd(q, kb, vb, num, idx, block)
    n, ix = num.cpu(), idx.cpu()
    lists = [[[ix[b, h, i, : n[b, h, i]].tolist() for i in range(n.shape[2])] for h in range(H)] for b in range(B)]
    check_attention(o, lse, q.cpu(), c, lists, [Lk] * B, 1 / math.sqrt(D))
    check_attention(o2, lse2, q.cpu(), c, lists, [Lk] * B, 1 / math.sqrt(D))
    # the values kept are the written ones to half a step of e4m3
    err = (kb.cpu().double() - k.double()).abs()
    amax = k.double().abs().amax()
    assert (err <= 2.0 ** -4 * k.double().abs() + 2.0 ** -17 * amax).all()


@pytest.mark.parametrize("Lq", [1, 100])
def test_token_loop_in_a_graph(gpu_lib, Lq):
    """Append and attend captured once; each replay appends at the device's own length."""
    S = gpu_lib
    D, block, B, H, cap, first = 128, 64, 2, 2, 4000, 3000
    g = torch.Generator().manual_seed(12)
    c = filled(S, g, B, H, cap, D, block)
    e = S.KvCache(*[t.clone() for t in c[:4]], block)
    k, v, q = (torch.empty(B, H, Lq, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    lens = torch.tensor([first, first - 70], dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
    ws = torch.empty(S.sparstar_cache_attn_workspace_bytes(B, H, Lq, cap, D, block), dtype=torch.uint8, device="cuda")

    def step(cache, lens):
        S.sparstar_cache_write(k, v, cache, starts=lens)
        lens.add_(Lq)
        S.sparstar_cache_dense_attn_fwd(q, cache, lens=lens, out=o, lse=lse, workspace=ws)

    def refill(i):
        gi = torch.Generator().manual_seed(100 + i)
        for t in (k, v, q):
            t.copy_(tokens(gi, B, H, Lq, D, 1.0))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    refill(0)
    with torch.cuda.stream(stream):
        step(S.KvCache(*[t.clone() for t in c[:4]], block), lens.clone())
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(c, lens)
    torch.cuda.synchronize()
    eager = lens.clone()
    for i in range(4):
        refill(i)
        step(e, eager)
        want = o.clone(), lse.clone()
        o.fill_(float("nan"))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _say(f"[cache graph] Lq={Lq} replay {i}")
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(lens, eager)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(c[:4], e[:4]))
        check_attention(o, lse, q.cpu(), c, None, lens.tolist(), 1 / math.sqrt(D))


def test_two_calls_at_once(gpu_lib):
    D, block, cap = 128, 64, 6000
    g = torch.Generator().manual_seed(13)
    runs = [(torch.randn(1, 2, Lq, D, generator=g).bfloat16().cuda(), filled(gpu_lib, g, 1, 2, cap, D, block))
            for Lq in (1, 300)]
    want = [gpu_lib.sparstar_cache_dense_attn_fwd(*r) for r in runs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in runs], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = gpu_lib.sparstar_cache_dense_attn_fwd(*runs[i])
    torch.cuda.synchronize()
    for w, t in zip(want, got):
        assert torch.equal(w[0], t[0]) and torch.equal(w[1], t[1])


def test_offsets_past_32_bits(gpu_lib):
    """Three heads of 2^24 rows: codes past 2^32 bytes are written, read and attended to."""
    S = gpu_lib
    D, block, H = 128, 64, 3
    cap = 1 << 24
    c = S.KvCache.empty(1, H, cap, D, block)
    for t in c[:4]:
        t.view(torch.uint8).fill_(127 if t.dtype == torch.uint8 else 0)
    _say(f"[cache long] {H} x {cap} rows")
    g = torch.Generator().manual_seed(14)
    L, Lq = 150, 2
    k, v = tokens(g, 1, H, L, D, 1.0), tokens(g, 1, H, L, D, 1.0)
    S.sparstar_cache_write(k.cuda(), v.cuda(), c, cap - L)
    kb, vb = S.sparstar_cache_read(c, cap - L, L)
    err = (kb.cpu().double() - k.double()).abs()
    # The first tokens continue a block whose scale byte is 127 (e = 0), and all values fit
    # below 448, so e <= 0 everywhere: half a step is at most 2^-4 of the value where its
    # code is normal, and 2^(e-10) <= 2^-10 where it is not.
    assert k.double().abs().amax() <= 448
    assert (err <= torch.maximum(2.0 ** -4 * k.double().abs(), torch.tensor(2.0 ** -10))).all()
    q = torch.randn(1, H, Lq, D, generator=g).bfloat16()
    n_k = cap // block
    for rows in (Lq, 40):
        q = torch.randn(1, H, rows, D, generator=g).bfloat16()
        num = torch.full((1, H, 1), 2, dtype=torch.int32, device="cuda")
        idx = torch.tensor([n_k - 2, n_k - 1], dtype=torch.int32, device="cuda").expand(1, H, 1, 2).contiguous()
        o, lse = S.sparstar_cache_sparse_attn_fwd(q.cuda(), c, num, idx)
        for h in range(H):
            kk, vv = kb[0, h, -128:].cpu().double(), vb[0, h, -128:].cpu().double()
            want = R.forward_tol(q[0, h].double(), kk, vv, torch.ones(rows, 128, dtype=torch.bool), 1 / math.sqrt(D))
            R.close(o[0, h], want[0], want[2], "o")
            R.close(lse[0, h], want[1], want[3], "lse")
