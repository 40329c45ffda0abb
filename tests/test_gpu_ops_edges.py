"""Calls of the gradients and the 8-bit cache that their documentation allows and that are easy
to get wrong: a fresh cache begun inside a block, O in place of Q, no lse, one buffer in two
roles, a workspace elsewhere."""
from __future__ import annotations

import math

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device
from tests.test_gpu_cache import check_attention, filled, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [64, 128])
def test_a_fresh_cache_may_begin_inside_a_block(gpu_lib, block):
    """Rows before the first written one are nobody's: whatever the buffers hold there, the
    new rows get the scale that they would get alone."""
    S = gpu_lib
    B, H, D, cap = 2, 2, 64, 300
    g = torch.Generator().manual_seed(block)
    junk = torch.full((1 << 20,), 0xff, dtype=torch.uint8, device="cuda")  # what a new cache may find
    del junk
    c = S.KvCache.empty(B, H, cap, D, block)
    k, v = tokens(g, B, H, 90, D), tokens(g, B, H, 90, D)
    starts = [5, 130]
    S.sparstar_cache_write(k.cuda(), v.cuda(), c, starts=torch.tensor(starts, dtype=torch.int32).cuda())
    ref = [R.RefCache(B, H, cap, D, block, torch.zeros(B, H, cap, D, dtype=torch.float64),
                      torch.zeros(B, H, -(-cap // block), dtype=torch.int64)) for _ in range(2)]
    for x, r in zip((k, v), ref):
        r.write(x.double(), starts)
    got = S.sparstar_cache_read(c, 0, cap)
    for t, r in zip(got, ref):
        want = r.values()
        for b, lo in enumerate(starts):
            assert torch.equal(t[b, :, lo:lo + 90].cpu().double(), want[b, :, lo:lo + 90])


@pytest.mark.parametrize("Lq,cap", [(1, 500), (3, 9000), (100, 500), (100, 9000)])
@pytest.mark.parametrize("sparse", [False, True])
def test_without_lse_and_in_place(gpu_lib, Lq, cap, sparse):
    S = gpu_lib
    D, block, B, H = 128, 64, 1, 2
    g = torch.Generator().manual_seed(Lq + cap)
    c = filled(S, g, B, H, cap, D, block)
    q = torch.randn(B, H, Lq, D, generator=g).bfloat16()
    lists = R.random_lists(g, B, H, -(-Lq // block), -(-cap // block), 0.5) if sparse else None
    listed = lists_to_device(lists, -(-Lq // block)) if sparse else ()
    call = S.sparstar_cache_sparse_attn_fwd if sparse else S.sparstar_cache_dense_attn_fwd
    o, lse = call(q.cuda(), c, *listed)
    check_attention(o, lse, q, c, lists, [cap], 1 / math.sqrt(D))
    o2, none = call(q.cuda(), c, *listed, return_lse=False)
    assert none is None and torch.equal(o2, o)
    qo = q.cuda()
    o3, lse3 = call(qo, c, *listed, out=qo)
    assert o3 is qo and torch.equal(qo, o) and torch.equal(lse3, lse)


def test_one_tensor_in_two_roles(gpu_lib):
    """K as V, Q as dO: inputs may share memory."""
    S = gpu_lib
    D, block, Lq, Lk = 64, 64, 130, 200
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn(1, 1, Lq, D, generator=g).bfloat16(), torch.randn(1, 1, Lk, D, generator=g).bfloat16()
    x = [q[0, 0].double(), k[0, 0].double(), k[0, 0].double()]
    mask = torch.ones(Lq, Lk, dtype=torch.bool)
    o64, l64, _ = R.forward(*x, mask, 1 / math.sqrt(D))
    qd, kd = q.cuda(), k.cuda()
    o, lse = R.rounded(o64)[None, None].cuda(), l64.float()[None, None].cuda()
    got = S.sparstar_dense_attn_bwd(qd, kd, kd, o, lse, qd, block)
    want, tol = R.backward(*x, mask, 1 / math.sqrt(D), q[0, 0].double())
    for t, w, e, name in zip(got, want, tol, ("dq", "dk", "dv")):
        R.close(t[0, 0], w, e, name)
    c = S.KvCache.empty(1, 1, Lk, D, block)
    S.sparstar_cache_write(kd, kd, c)
    assert torch.equal(c.k.view(torch.uint8), c.v.view(torch.uint8)) and torch.equal(c.k_scale, c.v_scale)


def test_a_workspace_elsewhere_is_refused(gpu_lib):
    S = gpu_lib
    q = torch.zeros(1, 1, 64, 64, dtype=torch.bfloat16, device="cuda")
    lse, far = torch.zeros(1, 1, 64, device="cuda"), torch.empty(1 << 24, dtype=torch.uint8)
    strided = torch.empty(1 << 12, 512, dtype=torch.uint8, device="cuda")[:, ::2]
    c = S.KvCache.empty(1, 1, 4096, 64, 64)
    for ws in (far, strided):
        with pytest.raises(ValueError):
            S.sparstar_dense_attn_bwd(q, q, q, q, lse, q, workspace=ws)
        with pytest.raises(ValueError):
            S.sparstar_cache_dense_attn_fwd(q, c, workspace=ws)


def test_nothing_of_infinite_or_nan_gradients_leaves_its_blocks(gpu_lib):
    """A row whose dO is NaN or infinite spoils its own dQ and the keys that it sees; a row
    without keys (lse = -inf) spoils nothing, whatever its dO, O and dlse hold."""
    S = gpu_lib
    D, block, Lq, Lk = 128, 64, 256, 320
    g = torch.Generator().manual_seed(5)
    q, do = (torch.randn(1, 1, Lq, D, generator=g).bfloat16() for _ in range(2))
    k, v = (torch.randn(1, 1, Lk, D, generator=g).bfloat16() for _ in range(2))
    lists = [[[[0, 2], [], [1, 2], [4]]]]
    num, idx = lists_to_device(lists, 4)
    o, lse = S.sparstar_sparse_attn_fwd(q.cuda(), k.cuda(), v.cuda(), num, idx, block)
    dlse = torch.zeros(1, 1, Lq)
    clean = S.sparstar_sparse_attn_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), num, idx, block,
                                       dlse=dlse.cuda())
    do[0, 0, 64:128], dlse[0, 0, 64:128], o[0, 0, 64:128] = math.nan, math.inf, -math.inf
    bad = S.sparstar_sparse_attn_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), num, idx, block,
                                     dlse=dlse.cuda())
    for a, b in zip(clean, bad):
        assert torch.equal(a, b)
    do[0, 0, 200] = math.inf  # a row of the last query block: key block 4 alone
    bad = S.sparstar_sparse_attn_bwd(q.cuda(), k.cuda(), v.cuda(), o, lse, do.cuda(), num, idx, block,
                                     dlse=dlse.cuda())
    keep = [r for r in range(Lq) if r != 200]
    assert torch.equal(bad[0][0, 0, keep], clean[0][0, 0, keep]) and not bad[0][0, 0, 200].isfinite().all()
    for a, b in zip(clean[1:], bad[1:]):
        assert torch.equal(a[0, 0, :256], b[0, 0, :256]) and not b[0, 0, 256:].isfinite().all()
