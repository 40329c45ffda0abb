"""GPU parity of the attention gradients against float64 (tests/grad_cache_ref.py), with
bounds per element derived from the roundings that the kernels make."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device
from tests.test_ops_abi import bwd_plan

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def make(seed, B, H, Lq, Lk, D, sharp=1.0, with_lse=False):
    g = torch.Generator().manual_seed(seed)
    q, do = (torch.randn(B, H, Lq, D, generator=g).bfloat16() for _ in range(2))
    k, v = (torch.randn(B, H, Lk, D, generator=g).bfloat16() for _ in range(2))
    q = (q.float() * sharp).bfloat16()
    return g, q, k, v, do, torch.randn(B, H, Lq, generator=g) if with_lse else None


def reference(q, k, v, do, dlse, lists, block, scale):
    """Per (b, h): o and lse (float64), the gradients and their bounds."""
    B, H, Lq, D = q.shape
    Lk = k.shape[2]
    out = {}
    for b in range(B):
        for h in range(H):
            mask = R.visible(lists[b][h] if lists is not None else None, Lq, Lk, block)
            x = [t[b, h].double() for t in (q, k, v)]
            dl = dlse[b, h].double() if dlse is not None else None
            o, lse, _ = R.forward(*x, mask, scale)
            out[b, h] = (o, lse, *R.backward(*x, mask, scale, do[b, h].double(), dl))
    return out


def run(S, q, k, v, do, dlse, lists, block, scale, ref):
    """The library's gradients, given the reference's o (rounded to bf16) and lse (fp32)."""
    B, H, Lq, D = q.shape
    o = torch.stack([torch.stack([R.rounded(ref[b, h][0]) for h in range(H)]) for b in range(B)]).cuda()
    lse = torch.stack([torch.stack([ref[b, h][1].float() for h in range(H)]) for b in range(B)]).cuda()
    args = [t.cuda() for t in (q, k, v)] + [o, lse, do.cuda()]
    dl = dlse.cuda() if dlse is not None else None
    sc = 0.0 if scale == 1 / math.sqrt(D) else scale
    if lists is None:
        return S.sparstar_dense_attn_bwd(*args, block, sc, dlse=dl)
    num, idx = lists_to_device(lists, -(-Lq // block))
    return S.sparstar_sparse_attn_bwd(*args, num, idx, block, sc, dlse=dl)


def check(grads, ref, B, H):
    for b in range(B):
        for h in range(H):
            for got, want, tol, name in zip(grads, ref[b, h][2], ref[b, h][3], ("dq", "dk", "dv")):
                R.close(got[b, h], want, tol, f"{name}[{b},{h}]")


CASES = [
    # D, block, B, H, Lq, Lk, lists (None: dense), density, sharp, scale factor, dlse
    (64, 64, 1, 1, 1, 1, None, 0, 1, 1, False),
    (128, 128, 1, 2, 1, 1, "full", 0, 1, 1, True),
    (128, 64, 1, 1, 63, 65, "full", 0, 1, 1, False),
    (64, 128, 2, 1, 65, 63, None, 0, 1, 1, True),
    (128, 64, 1, 2, 200, 517, "random", 0.4, 1, 1, False),
    (128, 128, 2, 2, 300, 700, "random", 0.5, 1, 1, True),
    (64, 64, 1, 3, 333, 401, "holes", 0.5, 1, 1, True),
    (64, 128, 1, 2, 257, 640, "random", 0.4, 2, 1, False),
    (128, 64, 1, 1, 129, 300, "one", 0, 1, 1, False),
    (128, 64, 1, 2, 320, 257, "holes", 0.3, 4, 1, False),
    (128, 64, 1, 2, 150, 333, None, 0, 4, 1, True),
    (64, 64, 2, 1, 130, 129, None, 0, 1, 0.01, False),
    (128, 128, 1, 1, 128, 256, None, 0, 0, 1, False),       # all logits equal
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"D{c[0]}b{c[1]}-{c[2]}x{c[3]}-{c[4]}x{c[5]}-{c[6]}")
def test_gradients_match_the_formula(gpu_lib, case):
    D, block, B, H, Lq, Lk, kind, density, sharp, factor, with_lse = case
    _say(f"[bwd] {case}")
    g, q, k, v, do, dlse = make(D + Lq + Lk, B, H, Lq, Lk, D, sharp, with_lse)
    scale = factor / math.sqrt(D)
    lists = R.random_lists(g, B, H, -(-Lq // block), -(-Lk // block), density, kind) if kind else None
    ref = reference(q, k, v, do, dlse, lists, block, scale)
    check(run(gpu_lib, q, k, v, do, dlse, lists, block, scale, ref), ref, B, H)


@pytest.mark.parametrize("D,block,Lq,Lk,dense", [(128, 64, 64, 2100, False), (128, 128, 100, 4200, True),
                                                 (64, 64, 40, 4200, False), (128, 64, 2100, 64, True),
                                                 (64, 128, 8300, 100, False), (128, 64, 4200, 128, False)])
def test_ranges_join(gpu_lib, D, block, Lq, Lk, dense):
    """Few work-groups: the keys of a row, or the queries of a key, are cut into ranges."""
    plan = bwd_plan(gpu_lib.load(), 1, 1, Lq, Lk, D, block, dense)
    _say(f"[bwd ranges] D={D} b={block} {Lq}x{Lk} dense={dense}: {plan}")
    assert max(plan) > 1
    g, q, k, v, do, dlse = make(Lq + Lk, 1, 1, Lq, Lk, D, 1, True)
    lists = None if dense else R.random_lists(g, 1, 1, -(-Lq // block), -(-Lk // block), 0.6, "holes")
    ref = reference(q, k, v, do, dlse, lists, block, 1 / math.sqrt(D))
    check(run(gpu_lib, q, k, v, do, dlse, lists, block, 1 / math.sqrt(D), ref), ref, 1, 1)


def test_more_query_blocks_than_a_batch_of_words(gpu_lib):
    """2,112 query blocks: a key block's words need more than one batch of 64."""
    D, block, Lq, Lk = 64, 64, 64 * 2111 + 5, 130
    _say(f"[bwd words] {Lq}x{Lk}")
    g, q, k, v, do, _ = make(3, 1, 1, Lq, Lk, D)
    lists = R.random_lists(g, 1, 1, -(-Lq // block), 3, 0.3, "holes")
    lists[0][0][-1] = [1, 2]
    ref = reference(q, k, v, do, None, lists, block, 1 / math.sqrt(D))
    check(run(gpu_lib, q, k, v, do, None, lists, block, 1 / math.sqrt(D), ref), ref, 1, 1)


def test_more_key_blocks_than_a_chunk_of_bits(gpu_lib):
    """8,200 key blocks: the bit matrix is built in more than one chunk."""
    D, block, Lq, Lk = 64, 64, 70, 64 * 8199 + 9
    _say(f"[bwd bits] {Lq}x{Lk}")
    g, q, k, v, do, _ = make(4, 1, 1, Lq, Lk, D)
    lists = [[[[0, 5, 8191, 8192, 8199], [8190, 8193, 8198]]]]
    ref = reference(q, k, v, do, None, lists, block, 1 / math.sqrt(D))
    check(run(gpu_lib, q, k, v, do, None, lists, block, 1 / math.sqrt(D), ref), ref, 1, 1)


def test_after_the_forward_and_against_differences(gpu_lib):
    """Selector, forward, gradient in a row, as a training step runs them.  The directional
    derivative that the gradients give is that of the float64 loss, by differences."""
    S = gpu_lib
    D, block, B, H, Lq, Lk = 128, 64, 1, 2, 200, 330
    g, q, k, v, do, dlse = make(17, B, H, Lq, Lk, D, 1, True)
    qd, kd, vd = (t.cuda() for t in (q, k, v))
    num, idx = S.sparstar_score_blocks(qd, kd, block, 0.5, [(0, 64)])
    o, lse = S.sparstar_sparse_attn_fwd(qd, kd, vd, num, idx, block)
    grads = S.sparstar_sparse_attn_bwd(qd, kd, vd, o, lse, do.cuda(), num, idx, block, dlse=dlse.cuda())
    torch.cuda.synchronize()
    n, ix = num.cpu(), idx.cpu()
    scale = 1 / math.sqrt(D)
    dirs = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (q, k, v)]

    def loss(step, which):
        total = 0.0
        for h in range(H):
            lists = [ix[0, h, i, : n[0, h, i]].tolist() for i in range(n.shape[2])]
            x = [t[0, h].double() + (step * d[0, h] if i == which else 0)
                 for i, (t, d) in enumerate(zip((q, k, v), dirs))]
            o64, l64, _ = R.forward(*x, R.visible(lists, Lq, Lk, block), scale)
            total += float((o64 * do[0, h].double()).sum() + (l64 * dlse[0, h].double()).sum())
        return total

    h = 1e-5
    for which, (got, d, name) in enumerate(zip(grads, dirs, ("dq", "dk", "dv"))):
        want = (loss(h, which) - loss(-h, which)) / (2 * h)
        prod = got.cpu().double() * d
        # independent roundings of each element's terms: three of at most 2^-8 of the
        # gradient's size, added as a random sum; six times its deviation
        tol = 6 * 3 * R.U * float(prod.square().sum().sqrt()) + 1e-6 * abs(want)
        _say(f"[bwd diff] {name}: {float(prod.sum()):.5f} want {want:.5f} tol {tol:.5f}")
        assert abs(float(prod.sum()) - want) <= tol, name


def test_shared_heads_as_one_head(gpu_lib):
    """Two query heads over one key head, as a view: dk and dv are the sums."""
    D, block, G, Lq, Lk = 64, 64, 2, 128, 200
    g, q, k, v, do, _ = make(21, 1, 1, G * Lq, Lk, D)
    lists = R.random_lists(g, 1, 1, G * Lq // block, -(-Lk // block), 0.5)
    ref = reference(q, k, v, do, None, lists, block, 1 / math.sqrt(D))
    grads = run(gpu_lib, q, k, v, do, None, lists, block, 1 / math.sqrt(D), ref)
    check(grads, ref, 1, 1)
    rows = Lq // block
    parts = [[lists[0][0][x * rows:(x + 1) * rows]] for x in range(G)]
    dk, tol = 0, 0
    for x in range(G):
        qs, dos = (t.view(1, G, Lq, D)[:, x:x + 1] for t in (q, do))
        r = reference(qs, k, v, dos, None, [parts[x]], block, 1 / math.sqrt(D))[0, 0]
        dk, tol = dk + r[2][1], tol + r[3][1]
    R.close(grads[1][0, 0], dk, tol, "dk of shared heads")


def test_malformed_lists_and_empty_rows(gpu_lib):
    """Counts past the stride or negative, entries outside [0, n_k): skipped, as in the
    forward; the rest is what the valid entries give."""
    D, block, Lq, Lk = 128, 64, 256, 300
    g, q, k, v, do, _ = make(23, 1, 1, Lq, Lk, D)
    valid = [[[[0, 2, 4], [1, 3], [], []]]]
    ref = reference(q, k, v, do, None, valid, block, 1 / math.sqrt(D))
    num = torch.tensor([[[9, 4, -3, 0]]], dtype=torch.int32).cuda()
    idx = torch.tensor([[[[0, 2, 4, 77], [-1, 1, 3, 5], [0, 1, 2, 3], [0, 1, 2, 3]]]], dtype=torch.int32).cuda()
    o, lse = R.rounded(ref[0, 0][0])[None, None].cuda(), ref[0, 0][1].float()[None, None].cuda()
    grads = gpu_lib.sparstar_sparse_attn_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), num, idx, block)
    check(grads, ref, 1, 1)
    assert not grads[0][0, 0, 128:].any()


def test_no_queries_gives_zero_key_gradients(gpu_lib):
    q = torch.empty(1, 2, 0, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.randn(1, 2, 70, 64, device="cuda").bfloat16()
    lse = torch.empty(1, 2, 0, device="cuda")
    num = torch.empty(1, 2, 0, dtype=torch.int32, device="cuda")
    idx = torch.empty(1, 2, 0, 1, dtype=torch.int32, device="cuda")
    for lists in (None, (num, idx)):
        out = (torch.empty_like(q), torch.full_like(k, 7.0), torch.full_like(k, 7.0))
        if lists is None:
            gpu_lib.sparstar_dense_attn_bwd(q, k, k, q, lse, q, 64, out=out)
        else:
            gpu_lib.sparstar_sparse_attn_bwd(q, k, k, q, lse, q, *lists, 64, out=out)
        torch.cuda.synchronize()
        assert not out[1].any() and not out[2].any()


def test_writes_only_its_outputs(gpu_lib):
    """Guard bands around the gradients stay as they were; two calls give the same bits."""
    D, block, B, H, Lq, Lk = 128, 64, 1, 2, 130, 333
    g, q, k, v, do, _ = make(29, B, H, Lq, Lk, D)
    lists = R.random_lists(g, B, H, 3, 6, 0.5)
    num, idx = lists_to_device(lists, 3)
    args = [t.cuda() for t in (q, k, v)]
    o, lse = gpu_lib.sparstar_sparse_attn_fwd(*args, num, idx, block)
    pad = 4096
    raw = [torch.full((t.numel() + 2 * pad,), 3.0, dtype=torch.bfloat16, device="cuda") for t in args]
    out = [r[pad:pad + t.numel()].view(t.shape) for r, t in zip(raw, args)]
    need = gpu_lib.sparstar_attn_bwd_workspace_bytes(B, H, Lq, Lk, D, block)
    ws = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    gpu_lib.sparstar_sparse_attn_bwd(*args, o, lse, do.cuda(), num, idx, block, out=out, workspace=ws[:need])
    first = [t.clone() for t in out]
    gpu_lib.sparstar_sparse_attn_bwd(*args, o, lse, do.cuda(), num, idx, block, out=out, workspace=ws[:need])
    torch.cuda.synchronize()
    for r, t, f in zip(raw, out, first):
        assert torch.equal(t, f) and t.isfinite().all()
        assert (r[:pad] == 3).all() and (r[pad + t.numel():] == 3).all()
    assert (ws[need:] == 0xff).all()


@pytest.mark.parametrize("dense", [False, True])
def test_graph_replays_match_eager(gpu_lib, dense):
    """Forward and gradient captured together, replayed with eager work in between."""
    S = gpu_lib
    D, block, B, H, Lq, Lk = 64, 64, 1, 2, 300, 2500
    g, q, k, v, do, _ = make(31, B, H, Lq, Lk, D)
    q, k, v, do = (t.cuda() for t in (q, k, v, do))
    num, idx = lists_to_device(R.random_lists(g, B, H, 5, 40, 0.4), 5)
    assert max(bwd_plan(S.load(), B, H, Lq, Lk, D, block, dense)) > 1
    o, lse = torch.empty_like(q), torch.empty(B, H, Lq, device="cuda")
    out = tuple(torch.empty_like(t) for t in (q, k, v))
    ws = torch.empty(S.sparstar_attn_bwd_workspace_bytes(B, H, Lq, Lk, D, block), dtype=torch.uint8, device="cuda")

    def step():
        if dense:
            S.sparstar_dense_attn_fwd(q, k, v, block, out=o, lse=lse, split=False)
            S.sparstar_dense_attn_bwd(q, k, v, o, lse, do, block, out=out, workspace=ws)
        else:
            S.sparstar_sparse_attn_fwd(q, k, v, num, idx, block, out=o, lse=lse, split=False)
            S.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, out=out, workspace=ws)

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
    for rep in range(3):
        for t in out:
            t.fill_(float("nan"))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _say(f"[bwd graph] dense={dense} replay {rep}")
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert math.isfinite(float(torch.randn(1 << 18, device="cuda").sum()))


def test_two_calls_at_once(gpu_lib):
    """Two streams, each with its own workspace (the binding's default)."""
    D, block, Lq, Lk = 128, 64, 500, 3000
    data = [make(s, 1, 2, Lq, Lk, D) for s in (41, 43)]
    want, streams = [], [torch.cuda.Stream() for _ in data]
    args = []
    for g, q, k, v, do, _ in data:
        q, k, v, do = (t.cuda() for t in (q, k, v, do))
        o, lse = gpu_lib.sparstar_dense_attn_fwd(q, k, v, block)
        args.append((q, k, v, o, lse, do))
        want.append(gpu_lib.sparstar_dense_attn_bwd(*args[-1], block))
    torch.cuda.synchronize()
    got = [None, None]
    for rep in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = gpu_lib.sparstar_dense_attn_bwd(*args[i], block)
    torch.cuda.synchronize()
    for w, t in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, t))


def test_offsets_past_32_bits(gpu_lib):
    """Keys of more than 2^32 bytes per head: the last block's gradients, and zeros where
    nothing is listed."""
    D, block, H, Lq = 128, 64, 2, 64
    Lk = (1 << 24) + 100
    _say(f"[bwd long] {Lk} keys")
    k = torch.zeros(1, H, Lk, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g, q, kt, vt, do, _ = make(47, 1, H, Lq, 100, D)
    k[:, :, -100:], v[:, :, -100:] = kt.cuda(), vt.cuda()
    n_k = -(-Lk // block)
    num = torch.full((1, H, 1), 2, dtype=torch.int32, device="cuda")
    idx = torch.tensor([n_k - 2, n_k - 1], dtype=torch.int32, device="cuda").expand(1, H, 1, 2).contiguous()
    args = (q.cuda(), k, v)
    o, lse = gpu_lib.sparstar_sparse_attn_fwd(*args, num, idx, block, split=False)
    grads = gpu_lib.sparstar_sparse_attn_bwd(*args, o, lse, do.cuda(), num, idx, block)
    torch.cuda.synchronize()
    lo = (n_k - 2) * block
    assert lo <= Lk - 100
    for h in range(H):
        x = [q[0, h].double(), k[0, h, lo:].cpu().double(), v[0, h, lo:].cpu().double()]
        want, tol = R.backward(*x, torch.ones(Lq, Lk - lo, dtype=torch.bool), 1 / math.sqrt(D), do[0, h].double())
        # (o here is the forward's: its P is rounded too, twice 2^-8 of sum P |v|)
        o64, _, p = R.forward(*x, torch.ones(Lq, Lk - lo, dtype=torch.bool), 1 / math.sqrt(D))
        more = 2 * R.U * (do[0, h].double().abs() * (p @ x[2].abs())).sum(dim=1, keepdim=True)
        extra = p * more / math.sqrt(D) * R.SLACK
        tol = (tol[0] + extra @ x[1].abs(), tol[1] + extra.t() @ x[0].abs(), tol[2])
        R.close(grads[0][0, h], want[0], tol[0], "dq")
        R.close(grads[1][0, h, lo:], want[1], tol[1], "dk")
        R.close(grads[2][0, h, lo:], want[2], tol[2], "dv")
        assert not grads[1][0, h, :lo].any() and not grads[2][0, h, :lo].any()
