"""Writes and reads of the 8-bit cache whose work-groups are launched in more than one row (of
up to 2^20).  Smaller calls on the same data are the reference, bit for bit."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_writes_of_many_blocks(gpu_lib):
    """A million work-groups and more, blocks begun anywhere, any count of new tokens."""
    S = gpu_lib
    B, H, D, cap, block, L, part = 1100, 256, 64, 80, 64, 20, 100
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(B, H, L, D, generator=g, device="cuda").mul_(3).exp_().bfloat16() for _ in range(2))
    assert 2 * B * H * ((L + block - 2) // block + 1) > 1 << 20
    starts = torch.randint(-3, cap - 10, (B,), generator=g, device="cuda", dtype=torch.int32)
    counts = torch.randint(-1, L + 2, (B,), generator=g, device="cuda", dtype=torch.int32)

    def fresh():
        c = S.KvCache.empty(B, H, cap, D, block)
        gc = torch.Generator(device="cuda").manual_seed(2)
        for t in c[:2]:  # (codes without NaN)
            t.view(torch.uint8).copy_(torch.randint(0, 127, t.shape, generator=gc, device="cuda", dtype=torch.uint8))
        for t in c[2:4]:
            t.copy_(torch.randint(100, 140, t.shape, generator=gc, device="cuda", dtype=torch.uint8))
        return c

    got, want = fresh(), fresh()
    S.sparstar_cache_write(k, v, got, starts=starts, counts=counts)
    for b in range(0, B, part):
        c = S.KvCache(*[t[b:b + part] for t in want[:4]], block)
        S.sparstar_cache_write(k[b:b + part], v[b:b + part], c, starts=starts[b:b + part], counts=counts[b:b + part])
    torch.cuda.synchronize()
    old = fresh()
    for a, w, o, name in zip(got, want, old, ("k", "v", "k_scale", "v_scale")):
        a, w, o = (t.view(torch.uint8) for t in (a, w, o))
        assert torch.equal(a, w) and not torch.equal(a, o), name


@pytest.mark.parametrize("want", [("k", "v"), ("v",)])
def test_reads_of_many_rows(gpu_lib, want):
    S = gpu_lib
    B, H, D, cap, block, start = 2, 20, 128, 900_000, 128, 77
    L = cap - start - 5
    assert B * H * L * D // 16 > 256 << 20
    g = torch.Generator(device="cuda").manual_seed(3)
    c = S.KvCache.empty(B, H, cap, D, block)
    for t in c[:2]:
        t.view(torch.uint8).copy_(torch.randint(0, 127, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in c[2:4]:
        t.copy_(torch.randint(100, 140, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    got = S.sparstar_cache_read(c, start, L, want=want)
    for lo in range(0, L, 100_001):
        n = min(100_001, L - lo)
        part = S.sparstar_cache_read(c, start + lo, n)
        for name, a, p in zip(("k", "v"), got, part):
            if name in want:
                assert torch.equal(a[:, :, lo:lo + n], p), (name, lo)
            else:
                assert a is None
