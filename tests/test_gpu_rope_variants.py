"""Tables of many rows, 16 to a thread, and turns of many rows of neighbouring pairs, three heads to
a thread."""
from __future__ import annotations

import pytest
import torch

from tests import paged_ref as P
from tests.test_gpu_rope import projection

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,axes,pairs,far,amp", [
    (33_001, 3, 64, 2 ** 30, 1.0), (50_003, 1, 40, 144_512, -1.5), (8192 * 256 + 777, 2, 1, 2 ** 31 - 1, 1.0),
    (140_000, 4, 16, 90_000, 1.0), (32_768, 1, 64, 10, 1.0)])
def test_tables_of_many_rows(gpu_lib, rows, axes, pairs, far, amp):
    print(f"[rope table] {rows} rows of {pairs} pairs", flush=True)
    assert rows >= 8192 * (256 // pairs)
    g = torch.Generator().manual_seed(rows)
    coords = torch.randint(-far, far, (rows, axes), generator=g).int()
    freq = gpu_lib.sparstar_rope_frequencies(pairs, 10_000.0, factor=2.0, length=4096)
    axis = [i % axes for i in range(pairs)]
    whole = torch.full((rows + 64, pairs, 2), 7.0, device="cuda")
    got = gpu_lib.sparstar_rope_table(coords.cuda(), freq, axis, amp, out=whole[:rows])
    torch.cuda.synchronize()
    assert (whole[rows:] == 7).all()
    x = coords[:, torch.tensor(axis)].double() * torch.tensor(freq, dtype=torch.float64)
    want = amp * torch.stack([x.cos(), x.sin()], dim=-1)
    # the angle in fp64 (here and there), and one rounding to fp32
    tol = 2.0 ** -24 * want.abs() + abs(amp) * (2.0 ** -50 * x.abs()[..., None] + 2.0 ** -40)
    worst = float(((got.cpu().double() - want).abs() / tol).max())
    print(f"  {worst:.3f} of the bound", flush=True)
    assert worst <= 1


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("D,pairs,inter,packed,B,H,L,given", [
    (64, 16, True, True, 2, 4, 1100, False), (128, 64, True, False, 1, 5, 1700, True), (128, 24, True, True, 3, 3, 911, True),
    (128, 40, False, True, 1, 5, 1700, True), (64, 32, False, False, 2, 7, 600, False), (64, 32, True, True, 1, 8193, 1, True)])
def test_turns_of_three_heads_a_thread(gpu_lib, D, pairs, inter, packed, B, H, L, given, back):
    print(f"[rope] D={D} pairs={pairs} {B}x{H}x{L} back={back}", flush=True)
    assert B * H * L >= 8192
    g = torch.Generator().manual_seed(L + D)
    table = P.random_table(g, L + 40, pairs)
    x = projection(g, B, H, L, D, packed)
    pos = torch.randint(0, L + 40, (B, L), generator=g) if given else (torch.arange(L) + 17).expand(B, L)
    call = gpu_lib.sparstar_rope_bwd if back else gpu_lib.sparstar_rope_fwd
    kw = dict(interleaved=inter, positions=pos.int().contiguous().cuda() if given else None)
    want = P.turn(x.cpu(), table[pos][:, None], pairs, inter, back)
    whole = torch.full((B, L, 3, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    call(x, table.cuda(), 17, out=whole[:, :, 2].transpose(1, 2), **kw)
    torch.cuda.synchronize()
    assert torch.equal(whole[:, :, 2].transpose(1, 2).cpu(), want) and (whole[:, :, :2] == 7).all()
    call(x, table.cuda(), 17, out=x, **kw)  # in place
    assert torch.equal(x.cpu(), want)
