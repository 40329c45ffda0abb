"""Sizes whose launches would need 2^32 threads: refused with a message, before any launch."""
import pytest

from paper_2608_10519_amd import sparstar as S
from tests.test_ops_abi import _attend, _bwd, lib  # noqa: F401  (a fixture)

HEADS = dict(B=1 << 16, H=1 << 8)  # 2^24 of them


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("over", [dict(Lq=1, Lk=1, D=64), dict(Lq=1, Lk=1, D=128),
                                  dict(B=1, H=1 << 10, Lq=1 << 18, Lk=64, D=128)])
def test_gradients_refuse_launches_of_too_many_threads(lib, dense, over):  # noqa: F811
    assert _bwd(lib, dense, ws_bytes=1 << 60, **{**HEADS, **over}) == S.ERR_INVALID_ARG
    assert "too many rows and heads" in S.last_error()


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("over", [dict(Lq=1, Lk=64, cap=64), dict(Lq=32, Lk=1, cap=1), dict(Lq=128, Lk=64, cap=64)])
def test_cache_attention_refuses_launches_of_too_many_threads(lib, dense, over):  # noqa: F811
    assert _attend(lib, dense, ws=None, **HEADS, **over) == S.ERR_INVALID_ARG
    assert "too many query rows and heads" in S.last_error()
