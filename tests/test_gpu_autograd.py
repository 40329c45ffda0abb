"""The README's autograd Function around the forward and its gradient call, as a training step
uses it."""
from __future__ import annotations

import os
import re

import pytest
import torch

from tests import grad_cache_ref as R
from tests.helpers import lists_to_device

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def readme_function(S):
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    scope = {"torch": torch, "S": S}
    exec(next(b for b in blocks if "class SparseAttention" in b), scope)
    return scope["SparseAttention"]


@pytest.mark.gpu
def test_the_function_of_the_readme(gpu_lib):
    S = gpu_lib
    D, block, B, H, Lq, Lk = 128, 64, 1, 2, 200, 330
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(B, H, n, D, generator=g).bfloat16().cuda().requires_grad_() for n in (Lq, Lk, Lk))
    num, idx = lists_to_device(R.random_lists(g, B, H, 4, 6, 0.5, "holes"), 4)
    attend = readme_function(S).apply
    o, lse = attend(q, k, v, num, idx, block)
    seen = lse > -1e30  # (rows without keys have lse = -inf)
    w, u = torch.randn(o.shape, generator=g).bfloat16().cuda(), torch.randn(lse.shape, generator=g).cuda() * seen

    def grads(loss):
        return torch.autograd.grad(loss, (q, k, v))

    def direct(do, dlse):
        with torch.no_grad():
            return S.sparstar_sparse_attn_bwd(q, k, v, o, lse, do, num, idx, block, dlse=dlse)

    zero, one = torch.zeros_like(lse), torch.ones_like(o)
    both = grads((attend(q, k, v, num, idx, block)[0].float() * w.float()).sum()
                 + (attend(q, k, v, num, idx, block)[1].masked_fill(~seen, 0.0) * u).sum())
    only_o, only_lse = direct(w, zero), direct(torch.zeros_like(o), u)
    for got, a, b, name in zip(both, only_o, only_lse, "qkv"):
        assert torch.equal(got, a + b), name  # (bf16 gradients of two uses of a leaf are added in bf16)
    o1, lse1 = attend(q, k, v, num, idx, block)
    for got, want, name in zip(grads(o1.sum()), direct(one, zero), "qkv"):  # an expanded gradient
        assert torch.equal(got, want), name
    assert not S.sparstar_sparse_attn_fwd(q, k, v, num, idx, block)[0].requires_grad


def test_the_readme_has_the_function():
    assert issubclass(readme_function(None), torch.autograd.Function)
