"""The README's autograd Function around the rotation and its gradient call, out of a fused
projection and into the attention."""
from __future__ import annotations

import os
import re

import pytest
import torch

from tests import paged_ref as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def readme_functions(S):
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    scope = {"torch": torch, "S": S}
    for name in ("Rotate", "SparseAttention"):
        exec(next(b for b in blocks if f"class {name}" in b), scope)
    return scope["Rotate"], scope["SparseAttention"]


@pytest.mark.gpu
@pytest.mark.parametrize("inter,pairs", [(False, 64), (True, 24)])
def test_a_projection_rotated_and_attended(gpu_lib, inter, pairs):
    S, B, H, L, D, block, start = gpu_lib, 2, 2, 150, 128, 64, 9
    g = torch.Generator().manual_seed(pairs)
    rotate, attend = (f.apply for f in readme_functions(S))
    table = P.random_table(g, L + start, pairs).cuda()
    qkv = torch.randn(B, L, 3, H, D, generator=g).bfloat16().cuda().requires_grad_()
    n = -(-L // block)
    num = torch.full((B, H, n), n, dtype=torch.int32, device="cuda")
    idx = torch.arange(n, dtype=torch.int32, device="cuda").expand(B, H, n, n).contiguous()
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    q, k, v = rotate(q, table, start, inter), rotate(k, table, start, inter), v.contiguous()
    o, lse = attend(q, k, v, num, idx, block)
    w = torch.randn(o.shape, generator=g).bfloat16().cuda()
    (got,) = torch.autograd.grad((o.float() * w.float()).sum(), qkv)

    with torch.no_grad():
        grads = S.sparstar_sparse_attn_bwd(q, k, v, o, lse, w, num, idx, block, dlse=torch.zeros_like(lse))
    rows = table.cpu()[start : start + L]
    want = torch.stack([P.turn(x.cpu(), rows, pairs, inter, True) if i < 2 else x.cpu() for i, x in enumerate(grads)])
    assert torch.equal(got.cpu(), want.permute(1, 3, 0, 2, 4))

    x = qkv.detach()[:, :, 0].transpose(1, 2).requires_grad_()
    (got,) = torch.autograd.grad(rotate(x, table, start, inter).sum(), x)  # (an expanded gradient)
    assert torch.equal(got.cpu(), P.turn(torch.ones(B, H, L, D).bfloat16(), rows, pairs, inter, True))


def test_the_readme_has_the_functions():
    assert all(issubclass(f, torch.autograd.Function) for f in readme_functions(None))
