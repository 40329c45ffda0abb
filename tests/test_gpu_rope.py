"""Rotary positions on the GPU: the table against float64, turns bit for bit."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_ref as P

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def projection(g, B, H, L, D, packed):
    """x [B, H, L, D] on the GPU, dense or the middle slice of a fused projection."""
    if not packed:
        return torch.randn(B, H, L, D, generator=g).bfloat16().cuda()
    return torch.randn(B, L, 3, H, D, generator=g).bfloat16().cuda()[:, :, 1].transpose(1, 2)


TURNS = [
    # D, pairs, interleaved, packed, B, H, L, positions, amplitude
    (64, 32, False, False, 1, 1, 1, False, 1.0),
    (128, 64, False, True, 2, 24, 1, True, 1.0),
    (128, 64, True, False, 1, 5, 77, False, 1.25),
    (64, 8, False, True, 3, 2, 33, True, 1.0),
    (64, 24, False, False, 2, 3, 129, True, 1.0),
    (64, 16, True, True, 2, 3, 200, False, 1.0),
    (128, 40, False, True, 1, 7, 515, True, 1.0),
    (128, 8, True, True, 1, 4, 50, True, 0.5),
    (128, 64, False, True, 1, 24, 3000, True, 1.0),
]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("case", TURNS, ids=lambda c: f"D{c[0]}p{c[1]}-{c[4]}x{c[5]}x{c[6]}")
def test_turns(gpu_lib, case, back):
    D, pairs, inter, packed, B, H, L, given, amp = case
    _say(f"[rope] {case} back={back}")
    g = torch.Generator().manual_seed(L + D)
    T = L + 40
    table = P.random_table(g, T, pairs, amp)
    x = projection(g, B, H, L, D, packed)
    pos = torch.randint(0, T, (B, L), generator=g) if given else (torch.arange(L) + 17).expand(B, L)
    call = gpu_lib.sparstar_rope_bwd if back else gpu_lib.sparstar_rope_fwd
    kw = dict(interleaved=inter, positions=pos.int().contiguous().cuda() if given else None)
    y = call(x, table.cuda(), 17, **kw)
    want = P.turn(x.cpu(), table[pos][:, None], pairs, inter, back)
    assert y.is_contiguous() and torch.equal(y.cpu(), want)
    # into a slice of a projection, whose other slices stay; and in place
    whole = torch.full((B, L, 3, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:, :, 2].transpose(1, 2)
    assert call(x, table.cuda(), 17, out=out, **kw) is out
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want) and (whole[:, :, :2] == 7).all()
    call(x, table.cuda(), 17, out=x, **kw)
    assert torch.equal(x.cpu(), want)


def test_nothing_outside_the_rows_is_written(gpu_lib):
    B, H, L, D = 2, 3, 45, 64
    g = torch.Generator().manual_seed(1)
    pad = torch.full((B * H * L * D + 512,), 9.0, dtype=torch.bfloat16, device="cuda")
    out = pad[256:-256].view(B, H, L, D)
    x = projection(g, B, H, L, D, False)
    gpu_lib.sparstar_rope_fwd(x, P.random_table(g, L, 32).cuda(), out=out)
    torch.cuda.synchronize()
    assert (pad[:256] == 9).all() and (pad[-256:] == 9).all()


@pytest.mark.parametrize("D,pairs,inter", [(128, 64, False), (64, 24, False), (128, 32, True)])
def test_gradient_against_differences(gpu_lib, D, pairs, inter):
    """The turn is linear: sum dy (f(x + h) - f(x)) = sum bwd(dy) h, up to the roundings of f
    (twice, 2^-8 of its values) and of the gradient (2^-8 of it)."""
    B, H, L = 2, 3, 50
    g = torch.Generator().manual_seed(5)
    table = P.random_table(g, L, pairs, 1.1).cuda()
    x, h, dy = (torch.randn(B, H, L, D, generator=g).bfloat16().cuda() for _ in range(3))
    x2 = (x.float() + h.float()).bfloat16()
    step = x2.double() - x.double()
    f = [gpu_lib.sparstar_rope_fwd(t, table, interleaved=inter).double() for t in (x, x2)]
    back = gpu_lib.sparstar_rope_bwd(dy, table, interleaved=inter).double()
    left, right = (dy.double() * (f[1] - f[0])).sum((1, 3)), (back * step).sum((1, 3))
    tol = 2.0 ** -8 * ((dy.double().abs() * (f[0].abs() + f[1].abs())).sum((1, 3)) + (back.abs() * step.abs()).sum((1, 3)))
    assert ((left - right).abs() <= tol).all()


def test_expanded_gradients_and_empty_calls(gpu_lib):
    g = torch.Generator().manual_seed(6)
    table = P.random_table(g, 9, 32)
    one = torch.ones((), dtype=torch.bfloat16, device="cuda").expand(2, 3, 9, 64)
    with pytest.raises(ValueError):  # (channels that are one and the same)
        gpu_lib.sparstar_rope_bwd(one, table.cuda())
    rows = torch.randn(64, generator=g).bfloat16().cuda().expand(2, 3, 9, 64)
    want = P.turn(rows.cpu(), table, 32, back=True)
    assert torch.equal(gpu_lib.sparstar_rope_bwd(rows, table.cuda()).cpu(), want)
    none = gpu_lib.sparstar_rope_fwd(rows[:, :, :0], table.cuda())
    assert none.shape == (2, 3, 0, 64)


def test_positions_outside_the_table_leave_the_others_right(gpu_lib):
    g = torch.Generator().manual_seed(7)
    table = P.random_table(g, 20, 32)
    x = torch.randn(1, 2, 30, 64, generator=g).bfloat16()
    pos = torch.randint(0, 20, (1, 30), generator=g)
    bad = torch.tensor([3, 11, 29])
    pos[0, bad] = torch.tensor([-1, 20, 2 ** 31 - 1])
    y = gpu_lib.sparstar_rope_fwd(x.cuda(), table.cuda(), positions=pos.int().cuda()).cpu()
    want = P.turn(x, table[pos.clamp(0, 19)][:, None], 32)
    keep = torch.ones(30, dtype=torch.bool)
    keep[bad] = False
    assert torch.equal(y[:, :, keep], want[:, :, keep])


def test_infinities_and_nan_stay_in_their_pairs(gpu_lib):
    g = torch.Generator().manual_seed(8)
    table = P.random_table(g, 4, 32)
    x = torch.randn(1, 1, 4, 128, generator=g).bfloat16()
    x[0, 0, 1, 3], x[0, 0, 2, 40], x[0, 0, 3, 100] = math.inf, math.nan, math.nan
    y = gpu_lib.sparstar_rope_fwd(x.cuda(), table.cuda()).cpu()
    want = P.turn(x, table, 32)
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y[~y.isnan()], want[~want.isnan()])
    assert y.isnan().sum() == 3 and y.isinf().sum() == 2


TABLES = [
    # rows, axes, pairs, largest coordinate, amplitude
    (1, 1, 1, 10, 1.0),
    (257, 1, 32, 144_512, 1.0),
    (1000, 3, 64, 90_000, 1.2),
    (513, 4, 40, 2 ** 30, 1.0),
    (300, 2, 64, 2 ** 31 - 1, -0.5),
]


@pytest.mark.parametrize("case", TABLES, ids=str)
def test_table(gpu_lib, case):
    rows, axes, pairs, far, amp = case
    _say(f"[rope table] {case}")
    g = torch.Generator().manual_seed(rows)
    coords = torch.randint(-far, far + 1 if far < 2 ** 31 - 1 else far, (rows, axes), generator=g).int()
    coords[0] = 0
    freq = gpu_lib.sparstar_rope_frequencies(pairs, 10_000.0, factor=2.0, length=4096)
    axis = [i % axes for i in range(pairs)]
    got = gpu_lib.sparstar_rope_table(coords.cuda(), freq, axis, amp).cpu().double()
    x = coords[:, torch.tensor(axis)].double() * torch.tensor(freq, dtype=torch.float64)
    want = amp * torch.stack([x.cos(), x.sin()], dim=-1)
    # the angle in fp64 (here and there), and one rounding to fp32
    tol = 2.0 ** -24 * want.abs() + abs(amp) * (2.0 ** -50 * x.abs()[..., None] + 2.0 ** -40)
    worst = ((got - want).abs() / tol).max()
    _say(f"  {float(worst):.3f} of the bound")
    assert worst <= 1
    assert torch.equal(got[0], (amp * torch.tensor([1.0, 0.0], dtype=torch.float64)).float().double().expand(pairs, 2))


def test_streams_devices_and_graphs(gpu_lib):
    """On a side stream and replayed from a graph, into a projection's gradient."""
    g = torch.Generator().manual_seed(9)
    B, H, L, D = 2, 4, 100, 128
    coords = torch.randint(0, 500, (L, 2), generator=g).int().cuda()
    freq, axis = gpu_lib.sparstar_rope_frequencies(64), [i // 32 for i in range(64)]
    x = projection(g, B, H, L, D, True)
    eager = gpu_lib.sparstar_rope_fwd(x, gpu_lib.sparstar_rope_table(coords, freq, axis))
    table, y = torch.empty(L, 64, 2, device="cuda"), torch.empty_like(eager)
    dqkv = torch.zeros(B, L, 3, H, D, dtype=torch.bfloat16, device="cuda")
    dx = dqkv[:, :, 0].transpose(1, 2)
    want_dx = gpu_lib.sparstar_rope_bwd(eager, gpu_lib.sparstar_rope_table(coords, freq, axis))

    def step():
        gpu_lib.sparstar_rope_table(coords, freq, axis, out=table)
        gpu_lib.sparstar_rope_fwd(x, table, out=y)
        gpu_lib.sparstar_rope_bwd(y, table, out=dx)

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(dx, want_dx)
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    for _ in range(3):
        table.zero_(), y.zero_(), dqkv.zero_()
        torch.randn(1 << 18, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(dx, want_dx) and (dqkv[:, :, 1:] == 0).all()


def test_more_work_groups_than_a_row_of_them(gpu_lib):
    """2^25 tokens: work-groups past 2^20, offsets past 2^32 bytes, in place."""
    L, D = (1 << 25) + 700, 64
    g = torch.Generator().manual_seed(12)
    table = P.random_table(g, 97, 32)
    pos = (torch.arange(L, dtype=torch.int32, device="cuda") % 97)[None].contiguous()
    x = torch.empty(1, 1, L, D, dtype=torch.bfloat16, device="cuda")
    rows = torch.randn(1, 1, 300, D, generator=g).bfloat16()
    at = [0, (1 << 25) - 150, L - 300]
    for i in at:
        x[:, :, i: i + 300] = rows.cuda()
    gpu_lib.sparstar_rope_fwd(x, table.cuda(), positions=pos, out=x)
    for i in at:
        assert torch.equal(x[:, :, i: i + 300].cpu(), P.turn(rows, table[torch.arange(i, i + 300) % 97], 32))
