"""The float64 references themselves: gradients against differences, the e4m3 grid and
rounding against torch's casts."""
import math

import pytest
import torch

from tests import grad_cache_ref as R


@pytest.mark.parametrize("with_lse", [False, True])
def test_reference_gradient_matches_differences(with_lse):
    g = torch.Generator().manual_seed(5)
    Lq, Lk, D, block = 9, 14, 6, 4
    q, k, v, do = (torch.randn(n, D, generator=g, dtype=torch.float64) for n in (Lq, Lk, Lk, Lq))
    dl = torch.randn(Lq, generator=g, dtype=torch.float64) if with_lse else None
    lists = [[0, 2], [], [1, 2, 3]]  # the second query block sees nothing
    mask, scale = R.visible(lists, Lq, Lk, block), 0.7

    def loss(q, k, v):
        o, lse, _ = R.forward(q, k, v, mask, scale)
        return float((o * do).sum() + (0 if dl is None else (lse * dl)[lse.isfinite()].sum()))

    grads, _ = R.backward(q, k, v, mask, scale, do, dl)
    if dl is not None:  # rows without keys have no lse
        assert not grads[0][4:8].any()
    h = 1e-6
    for x, gx in zip((q, k, v), grads):
        for _ in range(12):
            d = torch.randn(x.shape, generator=g, dtype=torch.float64)
            args = [q, k, v]
            at = next(i for i, t in enumerate(args) if t is x)
            up, down = ([t + s * h * d if i == at else t for i, t in enumerate(args)] for s in (1, -1))
            num = (loss(*up) - loss(*down)) / (2 * h)
            assert math.isclose(num, float((gx * d).sum()), rel_tol=1e-6, abs_tol=1e-7)


def test_e4m3_reference_matches_torch():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    want = codes.float().double()
    got = R.e4m3_values()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~got.isnan()], want[~want.isnan()])
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.linspace(-0.02, 0.02, 4001)]).float()
    assert torch.equal(R.e4m3_round(x.double()), x.to(torch.float8_e4m3fn).float().double())
    inf = R.e4m3_round(torch.tensor([math.inf, -math.inf, math.nan], dtype=torch.float64))
    assert inf[0] == 448 and inf[1] == -448 and inf[2].isnan()


@pytest.mark.parametrize("amax,e", [(0.0, -117), (448.0, 0), (448.0001, 1), (1.0, -8), (1.75, -8), (1.7500001, -7),
                                    (2.0 ** -130, -117), (3.3e38, 120)])
def test_scale_rule(amax, e):
    assert R.scale_exp(amax) == e
