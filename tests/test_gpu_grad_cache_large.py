"""The gradients and the attention over the 8-bit cache where there are many work-groups:
several rounds of them, key blocks of very different counts, lists walked from rotated
starts, pairs shared by XCDs.  Float64 on the GPU is the reference, one head at a time."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device
from tests.test_gpu_cache import filled, values_of
from tests.test_ops_abi import bwd_plan

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def lists_with_common_blocks(g, B, H, n_q, n_k, density, common):
    """Every row names the first `common` key blocks (as forced ones are), some name none."""
    out = R.random_lists(g, B, H, n_q, n_k, density)
    for b in range(B):
        for h in range(H):
            for i, row in enumerate(out[b][h]):
                out[b][h][i] = [] if i % 11 == 5 else sorted(set(row) | set(range(common)))
    return out


GRADS = [
    # D, block, B, H, Lq, Lk, density (None: dense), common blocks
    (128, 64, 1, 8, 2501, 5101, 0.2, 3),
    (64, 128, 2, 4, 2501, 8301, 0.2, 2),
    (128, 128, 2, 3, 3001, 4097, 0.3, 1),
    (64, 64, 2, 3, 1999, 3001, 0.3, 1),
    (128, 64, 2, 5, 1500, 4001, None, 0),
    # (each pass in a launch of its own)
    (128, 128, 2, 6, 1500, 6001, 0.3, 1),
    (64, 64, 2, 12, 1000, 4001, 0.3, 1),
    (128, 64, 2, 8, 1500, 6001, None, 0),
    (64, 64, 2, 8, 1500, 6001, None, 0),
    # (few key blocks, cut into many pieces; the last one of 60 keys)
    (64, 128, 1, 2, 9001, 700, 0.2, 2),
    (128, 64, 2, 1, 8200, 700, 0.2, 1),
    (128, 128, 1, 3, 5000, 2000, 1.0, 0),
]


@pytest.mark.parametrize("case", GRADS, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}-{c[4]}x{c[5]}-{c[6]}")
def test_gradients_of_many_work_groups(gpu_lib, case):
    D, block, B, H, Lq, Lk, density, common = case
    plan = bwd_plan(gpu_lib.load(), B, H, Lq, Lk, D, block, density is None)
    _say(f"[bwd large] {case}: {plan}")
    g = torch.Generator().manual_seed(Lq + Lk)
    q, do = (torch.randn(B, H, Lq, D, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(B, H, Lk, D, generator=g).bfloat16().cuda() for _ in range(2))
    dlse = torch.randn(B, H, Lq, generator=g).cuda()
    n_q, n_k, scale = -(-Lq // block), -(-Lk // block), 1 / math.sqrt(D)
    lists = None
    if density is not None:
        lists = lists_with_common_blocks(g, B, H, n_q, n_k, density, common)
        num, idx = lists_to_device(lists, n_q)
    masks, o, lse = {}, torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
    for b in range(B):
        for h in range(H):
            masks[b, h] = R.visible(lists[b][h] if lists is not None else None, Lq, Lk, block).cuda()
            x = [t[b, h].double() for t in (q, k, v)]
            o64, l64, _ = R.forward(*x, masks[b, h], scale)
            o[b, h], lse[b, h] = R.rounded(o64), l64.float()
    if lists is None:
        grads = gpu_lib.sparstar_dense_attn_bwd(q, k, v, o, lse, do, block, dlse=dlse)
    else:
        grads = gpu_lib.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, dlse=dlse)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(H):
            x = [t[b, h].double() for t in (q, k, v)]
            want, tol = R.backward(*x, masks[b, h], scale, do[b, h].double(), dlse[b, h].double())
            for got, w, t, name in zip(grads, want, tol, ("dq", "dk", "dv")):
                R.close(got[b, h], w.cpu(), t.cpu(), f"{name}[{b},{h}]")


@pytest.mark.parametrize("D,block,H,Lq,Lk", [(64, 128, 2, 6000, 700), (128, 64, 6, 2500, 9001)])
def test_cut_blocks_give_the_same_bits(gpu_lib, D, block, H, Lq, Lk):
    """Call after call, in a workspace of garbage, and in a graph that is replayed with eager
    work in between: the order in which blocks are listed changes nothing."""
    assert bwd_plan(gpu_lib.load(), 1, H, Lq, Lk, D, block, False)[1] > 1
    g = torch.Generator().manual_seed(Lq)
    q, do = (torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(1, H, Lk, D, generator=g).bfloat16().cuda() for _ in range(2))
    n_q, n_k = -(-Lq // block), -(-Lk // block)
    num, idx = lists_to_device(lists_with_common_blocks(g, 1, H, n_q, n_k, 0.1, 2), n_q)
    o, lse = gpu_lib.sparstar_sparse_attn_fwd(q, k, v, num, idx, block)
    out = tuple(torch.empty_like(t) for t in (q, k, v))
    need = gpu_lib.sparstar_attn_bwd_workspace_bytes(1, H, Lq, Lk, D, block)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        gpu_lib.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    for rep in range(4):
        for t in out:
            t.fill_(math.nan)
        ws.fill_(0x5a)
        torch.cuda.synchronize()
        graph.replay() if rep % 2 else step()
        torch.cuda.synchronize()
        _say(f"[bwd pieces] {Lq}x{Lk} {rep}")
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert math.isfinite(float(torch.randn(1 << 18, device="cuda").sum()))


def test_common_blocks_are_begun_first(gpu_lib):
    """The listed blocks' order is a matter of time alone: lists that are full give the
    dense call's dK and dV, whether key blocks count as common (a list's stride that is far
    above its entries says that they don't) or not."""
    D, block, H, Lq, Lk = 128, 64, 8, 1000, 5000
    g = torch.Generator().manual_seed(5)
    q, do = (torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(1, H, Lk, D, generator=g).bfloat16().cuda() for _ in range(2))
    n_q, n_k = -(-Lq // block), -(-Lk // block)
    # two thirds of the blocks on every list, the others on the first one alone
    rows = [list(range(n_k)) if i == 0 else list(range(2 * n_k // 3)) for i in range(n_q)]
    num = torch.tensor([len(r) for r in rows], dtype=torch.int32).expand(1, H, n_q).contiguous().cuda()
    idx = torch.full((n_q, n_k), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        idx[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
    wide = torch.full((1, H, n_q, 4 * n_k), -1, dtype=torch.int32, device="cuda")
    wide[..., :n_k] = idx.cuda()
    tight = wide[..., :n_k].contiguous()
    o, lse = gpu_lib.sparstar_sparse_attn_fwd(q, k, v, num, tight, block)
    a = gpu_lib.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, tight, block)
    b = gpu_lib.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, wide, block)
    for x, y, name in zip(a, b, ("dq", "dk", "dv")):
        assert torch.equal(x, y), name


ATTEND = [
    # D, block, B, H, Lq, cap, lens, density (None: dense), spread of the lists' lengths
    (128, 64, 1, 8, 5003, 6001, [6001], 0.25, False),
    (64, 64, 1, 12, 4003, 6001, [6001], 0.25, True),
    (128, 128, 2, 4, 4003, 6500, [6500, 2100], 0.3, True),
    (128, 64, 2, 12, 700, 7001, [7001, 33], 0.5, False),
    (64, 128, 1, 24, 2003, 4001, [4001], 1.0, False),
    (128, 64, 2, 6, 3003, 4001, [4001, 4000], None, False),
    # (few rows: up to 64 ranges)
    (128, 64, 1, 1, 64, 40_001, [40_001], None, False),
    (64, 128, 2, 1, 100, 70_001, [70_001, 777], 0.5, False),
    (128, 128, 1, 2, 190, 39_001, [0], None, False),
    (64, 64, 1, 1, 33, 33_000, [32_999], 0.9, True),
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}-{c[4]}x{c[5]}-{c[7]}")
def test_cache_attention_of_many_work_groups(gpu_lib, case):
    D, block, B, H, Lq, cap, lens, density, uneven = case
    _say(f"[cache large] {case}")
    g = torch.Generator().manual_seed(cap + Lq)
    c = filled(gpu_lib, g, B, H, cap, D, block)
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16().cuda()
    n_q, n_k = -(-Lq // block), -(-cap // block)
    lists = None
    if density is not None:
        lists = R.random_lists(g, B, H, n_q, n_k, density, "full" if density == 1.0 else "random")
        if uneven:  # heads of shorter and longer lists
            lists = [[[r[: max(1, len(r) * (h + 1) // H)] for r in rows] for h, rows in enumerate(heads)] for heads in lists]
    dl = None if set(lens) == {cap} else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if lists is None:
        o, lse = gpu_lib.sparstar_cache_dense_attn_fwd(q, c, lens=dl)
    else:
        o, lse = gpu_lib.sparstar_cache_sparse_attn_fwd(q, c, *lists_to_device(lists, n_q), lens=dl)
    kv = values_of(c)
    for b in range(B):
        m = lens[b]
        for h in range(H):
            mask = R.visible(lists[b][h] if lists is not None else None, Lq, cap, block)[:, :m].cuda()
            want = R.forward_tol(q[b, h].double(), kv[0][b, h, :m].cuda(), kv[1][b, h, :m].cuda(), mask,
                                 1 / math.sqrt(D))
            want = [t.cpu() for t in want]
            R.close(o[b, h], want[0], want[2], f"o[{b},{h}]")
            R.close(lse[b, h], want[1], want[3], f"lse[{b},{h}]")


def test_calls_follow_the_current_stream(gpu_lib):
    """Inputs made on a side stream, behind work that takes a while: every call goes to
    that stream too, and sees them."""
    S = gpu_lib
    D, block, H, L = 64, 64, 2, 700
    g = torch.Generator().manual_seed(6)
    host = [torch.randn(1, H, L, D, generator=g).bfloat16().pin_memory() for _ in range(4)]

    def step(q, k, v, do):
        c = S.KvCache.empty(1, H, L, D, block)
        S.sparstar_cache_write(k, v, c)
        kb, vb = S.sparstar_cache_read(c, 0, L)
        o, lse = S.sparstar_cache_dense_attn_fwd(q, c)
        return (o, lse, *S.sparstar_dense_attn_bwd(q, kb, vb, o, lse, do, block))

    want = step(*[t.cuda() for t in host])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = torch.randn(4096, 4096, device="cuda")
        data = [torch.full(t.shape, math.nan, dtype=t.dtype, device="cuda") for t in host]
        for _ in range(20):
            x = x @ x.clamp(-1e-2, 1e-2)
        for d, t in zip(data, host):
            d.copy_(t, non_blocking=True)
        got = step(*data)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
