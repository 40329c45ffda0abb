"""More refusals of the gradient and cache calls, without a GPU."""
import pytest
import torch

from paper_2608_10519_amd import sparstar as S
from tests.test_ops_abi import _attend, _bwd, _write, lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("dense", [False, True])
def test_gradients_refuse_a_scale_whose_inverse_leaves_fp32(lib, dense):  # noqa: F811
    assert _bwd(lib, dense, scale=1e-31) == S.ERR_INVALID_ARG
    assert "1e-30" in S.last_error()


def test_gradients_refuse_sizes_past_the_limits(lib):  # noqa: F811
    for over in (dict(Lk=1 << 40), dict(Lq=1 << 40)):
        assert _bwd(lib, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED), over
        assert S.last_error()


def test_cache_refuses_sizes_past_the_limits(lib):  # noqa: F811
    assert _write(lib, B=1 << 12, H=128, cap=1 << 28) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
    assert _attend(lib, Lq=1 << 40) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)


class Pretend(torch.Tensor):
    """A CPU tensor that says it is on the GPU: the binding's checks see it, nothing else."""

    is_cuda = True


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Pretend)


def test_binding_checks_shapes_types_and_layout():
    q, k = _t(1, 2, 8, 64), _t(1, 2, 16, 64)
    lse, num, idx = _t(1, 2, 8, dtype=torch.float32), _t(1, 2, 1, dtype=torch.int32), _t(1, 2, 1, 3, dtype=torch.int32)
    good = dict(v=k, o=q, lse=lse, d_o=q, num=num, idx=idx, dlse=None, out=None)
    for bad in (dict(v=_t(1, 2, 15, 64)), dict(v=_t(1, 2, 16, 64, dtype=torch.float16)), dict(o=k),
                dict(lse=lse.double().as_subclass(Pretend)), dict(d_o=_t(1, 2, 64, 8).transpose(2, 3)),
                dict(num=_t(1, 2, 2, dtype=torch.int32)), dict(idx=_t(1, 2, 3, dtype=torch.int32)),
                dict(dlse=_t(1, 2, 9, dtype=torch.float32)), dict(out=(q, k, q))):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            S.sparstar_sparse_attn_bwd(q, k, a["v"], a["o"], a["lse"], a["d_o"], a["num"], a["idx"], 64,
                                       dlse=a["dlse"], out=a["out"])
    cache = S.KvCache(_t(1, 2, 100, 64, dtype=torch.float8_e4m3fn), _t(1, 2, 100, 64, dtype=torch.float8_e4m3fn),
                      _t(1, 2, 2, dtype=torch.uint8), _t(1, 2, 2, dtype=torch.uint8), 64)
    for bad in (cache._replace(v=_t(1, 2, 99, 64, dtype=torch.float8_e4m3fn)), cache._replace(block_size=32),
                cache._replace(k_scale=_t(1, 2, 2, dtype=torch.int8)), cache._replace(block_size=0),
                cache._replace(k=_t(1, 2, 100, 64))):
        with pytest.raises(ValueError):
            S.sparstar_cache_dense_attn_fwd(q, bad)
        with pytest.raises(ValueError):
            S.sparstar_cache_write(k, k, bad)
    with pytest.raises(ValueError):
        S.sparstar_cache_write(k, k, cache, starts=_t(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.sparstar_cache_dense_attn_fwd(q, cache, lens=_t(1, dtype=torch.int64))
