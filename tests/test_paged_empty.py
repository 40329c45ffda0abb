"""Rotations and appends of no tokens with a table of no rows (the header asks for rows where
there are tokens)."""
import pytest
import torch

from paper_2608_10519_amd import sparstar as S
from tests.test_paged_abi import FAKE, _rope, _write, lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("table", [None, FAKE])
def test_no_tokens_need_no_table_rows(lib, back, table):  # noqa: F811
    assert _rope(lib, back, L=0, x=None, y=None, table=table, rows=0, start=0) == S.OK
    assert _write(lib, L=0, k=None, v=None, table=table, rows=0, start=0) == S.OK
    assert _write(lib, L=0, k=None, v=None, table=table, rows=0, starts=FAKE) == S.OK


def test_what_stays_refused(lib):  # noqa: F811
    for over in (dict(rows=-1, L=0), dict(rows=0, start=0), dict(rows=2 ** 40 + 1, L=0)):
        assert _rope(lib, **over) == S.ERR_INVALID_ARG and "table_rows" in S.last_error()
        assert _write(lib, **over) == S.ERR_INVALID_ARG and "table_rows" in S.last_error()
    assert _rope(lib, L=0, rows=0, start=1) == S.ERR_INVALID_ARG and "inside the table" in S.last_error()
    assert _write(lib, rows=0, starts=FAKE) == S.ERR_INVALID_ARG and "table_rows" in S.last_error()


@pytest.mark.gpu
def test_empty_tensors(gpu_lib):
    S, dev = gpu_lib, dict(device="cuda")
    x, pages = torch.empty(1, 2, 0, 64, dtype=torch.bfloat16, **dev), torch.zeros(1, 2, dtype=torch.int32, **dev)
    table = S.sparstar_rope_table(torch.empty(0, 1, dtype=torch.int32, **dev), [1.0] * 32)
    assert table.shape == (0, 32, 2)
    assert S.sparstar_rope_fwd(x, table).shape == S.sparstar_rope_bwd(x, table).shape == x.shape
    c = S.PagedCache.empty(2, 2, 64, 64)
    held = [t.clone() for t in c]
    S.sparstar_paged_write(x, x, c, pages, table=table)
    S.sparstar_paged_write(x, x, c, pages, table=table, positions=torch.empty(1, 0, dtype=torch.int32, **dev))
    assert all(torch.equal(a, b) for a, b in zip(c, held))
