"""How the sparse dK/dV pass orders and cuts its key blocks: what the list in the workspace
says, and that the gradients do not depend on it."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device

pytestmark = pytest.mark.gpu


def pieces_plan(lib, B, H, Lq, Lk, D, block, stride):
    """(list_min, piece_max, bytes before the list's length, bytes before its entries)"""
    out = (ctypes.c_int64 * 4)()
    i64 = ctypes.c_int64
    lib.sparstar_internal_bwd_pieces(B, H, i64(Lq), i64(Lk), D, block, i64(stride), out)
    return tuple(out)


def listed_pieces(ws, plan):
    """The list that a call left in its workspace: rows of block, piece, pieces, slot, begin, end."""
    n = int(ws[plan[2]:plan[2] + 4].view(torch.int32)[0])
    return ws[plan[3]:plan[3] + 32 * n].view(torch.int32).view(n, 8)[:, :6].cpu().tolist()


def runs(n_q, n_k, most):
    """Key block j is on the lists of neighbouring query blocks, a run that gets longer with j
    (up to `most`) and starts anywhere in a word of 32; the last block is on every list."""
    rows = [[] for _ in range(n_q)]
    for j in range(n_k):
        n = n_q if j == n_k - 1 else 1 + (most - 1) * j // max(1, n_k - 2)
        lo = 0 if j == n_k - 1 else 37 * j % (n_q - n + 1)
        for i in range(lo, lo + n):
            rows[i].append(j)
    return rows


def gradients_match(grads, q, k, v, do, lists, block, scale):
    B, H, Lq, _ = q.shape
    for b in range(B):
        for h in range(H):
            mask = R.visible(lists[b][h], Lq, k.shape[2], block).cuda()
            x = [t[b, h].double() for t in (q, k, v)]
            want, tol = R.backward(*x, mask, scale, do[b, h].double())
            for got, w, t, name in zip(grads, want, tol, ("dq", "dk", "dv")):
                R.close(got[b, h], w.cpu(), t.cpu(), f"{name}[{b},{h}]")


def forward64(q, k, v, lists, block, scale):
    B, H, Lq, _ = q.shape
    o, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
    for b in range(B):
        for h in range(H):
            mask = R.visible(lists[b][h], Lq, k.shape[2], block).cuda()
            o64, l64, _ = R.forward(*(t[b, h].double() for t in (q, k, v)), mask, scale)
            o[b, h], lse[b, h] = R.rounded(o64), l64.float()
    return o, lse


@pytest.mark.parametrize("D,block,H,Lq,Lk,most", [
    (64, 64, 2, 9001, 700, 90),
    (128, 128, 1, 6200, 2000, 30),
    (64, 64, 1, 64 * 700 + 3, 330, 650),  # 22 words per key block
])
def test_neighbouring_lists_are_cut_evenly(gpu_lib, D, block, H, Lq, Lk, most):
    """A piece has no more lists than the plan allows, also where the query blocks that list a
    key block are neighbours."""
    S = gpu_lib
    n_q, n_k = -(-Lq // block), -(-Lk // block)
    g = torch.Generator().manual_seed(Lq)
    q, do = (torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(1, H, Lk, D, generator=g).bfloat16().cuda() for _ in range(2))
    lists = [[runs(n_q, n_k, most) for _ in range(H)]]
    num, idx = lists_to_device(lists, n_q)
    scale = 1 / math.sqrt(D)
    o, lse = forward64(q, k, v, lists, block, scale)
    plan = pieces_plan(S.load(), 1, H, Lq, Lk, D, block, idx.shape[-1])
    need = S.sparstar_attn_bwd_workspace_bytes(1, H, Lq, Lk, D, block)
    ws = torch.full((need,), 0x5a, dtype=torch.uint8, device="cuda")
    grads = S.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, workspace=ws)
    torch.cuda.synchronize()
    got = listed_pieces(ws, plan)
    print(f"[bwd pieces] {H} x {Lq}x{Lk}: plan {plan[:2]}, {len(got)} pieces", flush=True)
    per_block = {}
    for blk, piece, pieces, slot, begin, end in got:
        per_block.setdefault(blk, []).append((piece, pieces, slot, begin, end))
    assert max(len(p) for p in per_block.values()) > 1
    slots = []
    for blk, found in per_block.items():
        found.sort()
        on = [i for i, row in enumerate(lists[0][blk // n_k]) if blk % n_k in row]
        pieces = -(-len(on) // plan[1])
        assert [f[:2] for f in found] == [(p, pieces) for p in range(pieces)]
        # one behind the other, from the first query block to the last
        assert found[0][3] == 0 and found[-1][4] == n_q
        assert all(a[4] == b[3] for a, b in zip(found, found[1:]))
        have = [sum(begin <= i < end for i in on) for *_, begin, end in found]
        assert sum(have) == len(on) and max(have) <= plan[1] and max(have) - min(have) <= 1, (blk, have)
        if pieces > 1:
            slots += [f[2] for f in found]
            assert [f[2] - found[0][2] for f in found] == list(range(pieces))
    assert sorted(slots) == list(range(len(slots)))
    assert set(per_block) >= {h * n_k + n_k - 1 for h in range(H)}
    gradients_match(grads, q, k, v, do, lists, block, scale)
    again = S.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("D,block,H,Lq,Lk", [(128, 64, 8, 1000, 5000), (64, 128, 9, 1300, 9001)])
def test_blocks_on_many_lists_are_begun_first(gpu_lib, D, block, H, Lq, Lk):
    """Blocks on more than twice the average count of lists come first, or all in order where
    the stride says that no count is far above it: the same bits, and float64's values."""
    S = gpu_lib
    n_q, n_k = -(-Lq // block), -(-Lk // block)
    g = torch.Generator().manual_seed(Lk)
    q, do = (torch.randn(1, H, Lq, D, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(1, H, Lk, D, generator=g).bfloat16().cuda() for _ in range(2))
    lists = R.random_lists(g, 1, H, n_q, n_k, 0.1)
    for rows in lists[0]:
        for i, row in enumerate(rows):
            rows[i] = sorted(set(row[:9]) | {0, n_k // 2, n_k - 1})  # three blocks on every list
    num, idx = lists_to_device(lists, n_q)
    assert idx.shape[-1] <= 12
    few = torch.full((1, H, n_q, 12), -1, dtype=torch.int32, device="cuda")
    many = torch.full((1, H, n_q, n_k), -1, dtype=torch.int32, device="cuda")
    few[..., :idx.shape[-1]] = many[..., :idx.shape[-1]] = idx
    scale = 1 / math.sqrt(D)
    o, lse = forward64(q, k, v, lists, block, scale)
    need = S.sparstar_attn_bwd_workspace_bytes(1, H, Lq, Lk, D, block)
    grads = []
    for stride, listed in ((few, True), (many, False)):
        plan = pieces_plan(S.load(), 1, H, Lq, Lk, D, block, stride.shape[-1])
        # three blocks of each head have n_q lists, and no block has more
        assert (0 < plan[0] < n_q) if listed else plan[0] >= n_q
        assert plan[1] >= n_q  # nothing is cut
        ws = torch.full((need,), 0x5a, dtype=torch.uint8, device="cuda")
        grads.append(S.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, stride, block, workspace=ws))
        torch.cuda.synchronize()
        found = listed_pieces(ws, plan)
        print(f"[bwd order] {H} x {Lq}x{Lk}: plan {plan[:2]}, {len(found)} listed", flush=True)
        if listed:
            assert {f[0] for f in found} >= {h * n_k + j for h in range(H) for j in (0, n_k // 2, n_k - 1)}
            assert len(found) < H * n_k // 2 and all(f[1:3] == [0, 1] for f in found)
        else:
            assert not found
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    gradients_match(grads[0], q, k, v, do, lists, block, scale)
