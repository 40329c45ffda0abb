"""Refusals of the rotary and paged-cache entry points and of their binding, and the host-side
frequencies: without a GPU (the fake device pointers are never dereferenced)."""
import ctypes
import math
import os

import pytest
import torch

from paper_2608_10519_amd import sparstar as S
from tests.test_ops_values import _t

FAKE = 0x10000
I32, U8, F32 = torch.int32, torch.uint8, torch.float32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.fail("libsparstar.so is not built (run __graft_entry__.build())")
    return S.load()


def dense(H, L, D):
    return S.Strides(H * L * D, L * D, D)


# ---- frequencies
def test_frequencies():
    assert S.sparstar_rope_frequencies(4, 16.0) == [1.0, 0.5, 0.25, 0.125]
    plain = S.sparstar_rope_frequencies(64)
    assert all(math.isclose(f, 10_000 ** (-p / 64), rel_tol=1e-15) for p, f in enumerate(plain))
    assert S.sparstar_rope_frequencies(64, factor=1.0, length=-5, slow=9, fast=2) == plain
    long = S.sparstar_rope_frequencies(64, factor=4.0, length=4096, slow=1, fast=32)
    for f, s in zip(plain, long):
        turns = 4096 * f / (2 * math.pi)
        if turns >= 32:
            assert s == f
        elif turns <= 1:
            assert math.isclose(s, f / 4, rel_tol=1e-15)
        else:
            g = (turns - 1) / 31
            assert math.isclose(s, g * f + (1 - g) * f / 4, rel_tol=1e-14)
    assert long[0] == plain[0] and math.isclose(long[-1], plain[-1] / 4, rel_tol=1e-15)


@pytest.mark.parametrize("over", [dict(pairs=0), dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(factor=0.5),
                                  dict(factor=math.nan), dict(factor=math.inf), dict(length=0.0), dict(length=math.inf),
                                  dict(slow=-1.0), dict(fast=1.0), dict(fast=math.inf), dict(slow=math.nan)])
def test_frequencies_refuse(lib, over):
    a = dict(pairs=8, base=1e4, factor=2.0, length=100.0, slow=1.0, fast=32.0)
    a.update(over)
    out = (ctypes.c_double * 8)()
    assert lib.sparstar_rope_frequencies(*a.values(), out) == S.ERR_INVALID_ARG and S.last_error()
    assert lib.sparstar_rope_frequencies(8, 1e4, 1.0, 0, 0, 0, None) == S.ERR_INVALID_ARG


# ---- table
def _table(lib, freq=(1.0, 0.1), axis=(0, 1), **over):
    a = dict(coords=FAKE, rows=10, axes=2, pairs=2, freq=(ctypes.c_double * 64)(*freq) if freq else None,
             axis=(ctypes.c_int32 * 64)(*axis) if axis else None, amp=1.0, table=FAKE)
    a.update(over)
    return lib.sparstar_rope_table(*a.values(), None)


@pytest.mark.parametrize("over,msg", [
    (dict(rows=-1), "rows"), (dict(axes=0), "axes"), (dict(axes=5), "axes"), (dict(pairs=0), "pairs"),
    (dict(pairs=65), "pairs"), (dict(freq=None), "freq"), (dict(amp=math.nan), "amplitude"), (dict(amp=math.inf), "amplitude"),
    (dict(freq=(1.0, math.nan)), "finite"), (dict(freq=(math.inf, 1.0)), "finite"), (dict(freq=(2.0 ** 21, 1.0)), "2^20"),
    (dict(axis=(0, 2)), "axis"), (dict(axis=(-1, 0)), "axis"), (dict(coords=None), "non-null"), (dict(table=None), "non-null"),
    (dict(coords=FAKE + 2), "aligned"), (dict(table=FAKE + 4), "aligned"),
])
def test_table_refuses(lib, over, msg):
    assert _table(lib, **over) == S.ERR_INVALID_ARG
    assert msg in S.last_error()


def test_table_of_nothing(lib):
    assert _table(lib, rows=0, coords=None, table=None) == S.OK


# ---- rotations
def _rope(lib, back=False, **over):
    a = dict(x=FAKE, xs=dense(2, 9, 64), B=3, H=2, L=9, D=64, table=FAKE, rows=20, pairs=32, inter=0, pos=None, start=11,
             y=FAKE + 4096, ys=dense(2, 9, 64))
    a.update(over)
    return (lib.sparstar_rope_bwd if back else lib.sparstar_rope_fwd)(*a.values(), None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("over,msg", [
    (dict(D=96), "head dim"), (dict(B=0), "B and H"), (dict(L=-1), "Lq"), (dict(pairs=0), "pairs"), (dict(pairs=12), "pairs"),
    (dict(pairs=40), "pairs"), (dict(rows=0), "table_rows"), (dict(start=12), "inside the table"),
    (dict(start=-1), "inside the table"), (dict(start=2 ** 62), "inside the table"), (dict(x=None), "non-null"),
    (dict(y=None), "non-null"), (dict(table=None), "non-null"), (dict(x=FAKE + 8), "16-byte"), (dict(y=FAKE + 2), "16-byte"),
    (dict(table=FAKE + 8), "16-byte"), (dict(pos=FAKE + 2), "4-byte"), (dict(xs=S.Strides(1152, 576, 60)), "multiples"),
    (dict(xs=S.Strides(-1152, 576, 64)), "negative"), (dict(ys=S.Strides(0, 576, 64)), "overlap"),
    (dict(ys=S.Strides(1152, 576, 56)), "overlap"), (dict(ys=S.Strides(1152, 512, 64)), "overlap"),
    (dict(xs=S.Strides(2 ** 60, 576, 64)), "too large"), (dict(xs=S.Strides(2 ** 46 - 8, 576, 64)), "too large"),
    (dict(y=FAKE, ys=S.Strides(1152, 64, 128)), "same strides"),
])
def test_rotations_refuse(lib, back, over, msg):
    assert _rope(lib, back, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
    assert msg in S.last_error()


def test_rotation_of_nothing(lib):
    assert _rope(lib, L=0, x=None, y=None, start=20) == S.OK
    assert _rope(lib, L=0, x=None, y=None, ys=S.Strides(0, 0, 64)) == S.OK  # as a dense tensor without tokens has them
    # strides of sizes of one do not matter
    assert _rope(lib, B=1, H=1, L=0, xs=S.Strides(-3, 7, 5), ys=S.Strides(1, 2, 3), x=None, y=None) == S.OK


# ---- the paged cache
def _write(lib, **over):
    a = dict(k=FAKE, ks=dense(2, 5, 64), v=FAKE, vs=dense(2, 5, 64), B=1, H=2, L=5, D=64, block=64, start=3, starts=None,
             counts=None, table=FAKE, rows=128, pairs=32, inter=0, pos=None, pages=FAKE, n_table=2, n_pages=4, kp=FAKE, vp=FAKE,
             ks2=FAKE, vs2=FAKE)
    a.update(over)
    return lib.sparstar_paged_write(*a.values(), None)


def _read(lib, **over):
    a = dict(kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, B=1, H=2, start=3, L=5, D=64, block=64, pages=FAKE, n_table=2, n_pages=4,
             k=FAKE, v=FAKE)
    a.update(over)
    return lib.sparstar_paged_read(*a.values(), None)


def _attend(lib, is_dense=False, **over):
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, B=1, H=2, Lq=5, Lk=128, D=64, block=64, pages=FAKE, n_table=2,
             n_pages=4, lens=None, num=FAKE, idx=FAKE, stride=2, scale=0.0, o=FAKE, lse=FAKE, ws=None, ws_bytes=0)
    a.update(over)
    if is_dense:
        for x in ("num", "idx", "stride"):
            a.pop(x)
        return lib.sparstar_paged_dense_attn_fwd(*a.values(), None)
    return lib.sparstar_paged_sparse_attn_fwd(*a.values(), None)


POOL = [(dict(D=96), "head dim"), (dict(block=32), "block size"), (dict(H=0), "B and H"), (dict(n_table=0), "n_table"),
        (dict(n_table=2 ** 30), "n_table"), (dict(n_pages=0), "n_pages"), (dict(n_pages=2 ** 31), "n_pages"),
        (dict(n_pages=2 ** 31 - 1, H=1000), "cache too large"), (dict(kp=None), "non-null"), (dict(pages=None), "non-null"),
        (dict(kp=FAKE + 8), "16-byte"), (dict(pages=FAKE + 2), "4-byte")]


@pytest.mark.parametrize("over,msg", POOL)
def test_a_malformed_pool_is_refused(lib, over, msg):
    for call in (_write, _read, _attend, lambda lib, **o: _attend(lib, True, **o)):
        assert call(lib, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
        assert msg in S.last_error()


@pytest.mark.parametrize("over,msg", [
    (dict(L=-1), "Lq"), (dict(start=-1), "pages' table"), (dict(start=124), "pages' table"),
    (dict(start=2 ** 63 - 1), "pages' table"), (dict(k=None), "non-null"), (dict(v=FAKE + 2), "16-byte"),
    (dict(starts=FAKE + 2), "4-byte"), (dict(counts=FAKE + 1), "4-byte"), (dict(ks2=FAKE + 4), "16-byte"),
    (dict(vs2=None), "non-null"), (dict(table=None, pos=FAKE), "without a table"), (dict(rows=7), "inside the table"),
    (dict(pairs=12), "pairs"), (dict(pairs=40), "pairs"), (dict(table=FAKE + 8), "16-byte"), (dict(pos=FAKE + 2), "4-byte"),
    (dict(ks=S.Strides(640, 324, 64)), "multiples"), (dict(vs=S.Strides(640, 320, -64)), "negative"),
])
def test_paged_write_refuses(lib, over, msg):
    assert _write(lib, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
    assert msg in S.last_error()


@pytest.mark.parametrize("over,msg", [(dict(start=-1), "pages' table"), (dict(start=124), "pages' table"), (dict(L=-1), "Lq"),
                                      (dict(k=FAKE + 8), "16-byte"), (dict(L=2 ** 62), "2^30")])
def test_paged_read_refuses(lib, over, msg):
    assert _read(lib, **over) == S.ERR_INVALID_ARG
    assert msg in S.last_error()


def test_paged_calls_of_nothing(lib):
    assert _write(lib, L=0, k=None, v=None, start=128) == S.OK
    assert _read(lib, L=0, start=128) == S.OK
    assert _read(lib, k=None, v=None) == S.OK
    assert _attend(lib, Lq=0, q=None, o=None, num=None) == S.OK


@pytest.mark.parametrize("is_dense", [False, True])
@pytest.mark.parametrize("over,code,msg", [
    (dict(Lk=129), S.ERR_INVALID_ARG, "Lk exceeds"), (dict(Lk=0), S.ERR_INVALID_ARG, "Lk"),
    (dict(Lq=-1), S.ERR_INVALID_ARG, "Lq"), (dict(Lq=1 << 40), S.ERR_INVALID_ARG, "2^30"),
    (dict(q=None), S.ERR_INVALID_ARG, "non-null"), (dict(o=FAKE + 8), S.ERR_INVALID_ARG, "16-byte"),
    (dict(lse=FAKE + 2), S.ERR_INVALID_ARG, "4-byte"), (dict(lens=FAKE + 2), S.ERR_INVALID_ARG, "4-byte"),
    (dict(scale=math.nan), S.ERR_INVALID_ARG, "finite"), (dict(scale=math.inf), S.ERR_INVALID_ARG, "finite"),
    (dict(ws=FAKE + 16, ws_bytes=1 << 40), S.ERR_WORKSPACE, "256-byte"),
    (dict(B=1 << 16, H=1 << 8, Lq=512), S.ERR_INVALID_ARG, "too many"),
])
def test_paged_attention_refuses(lib, is_dense, over, code, msg):
    assert _attend(lib, is_dense, **over) == code
    assert msg in S.last_error()


@pytest.mark.parametrize("over,msg", [(dict(num=None), "kv_num_blocks"), (dict(idx=None), "kv_indices"),
                                      (dict(stride=0), "kv_stride"), (dict(stride=(1 << 28) + 1), "kv_stride")])
def test_sparse_paged_attention_refuses_lists(lib, over, msg):
    assert _attend(lib, **over) == S.ERR_INVALID_ARG
    assert msg in S.last_error()


def test_workspaces(lib):
    """A workspace is asked for where a call may be cut, and has to be that large."""
    size = S.sparstar_paged_attn_workspace_bytes
    assert size(1, 2, 5, 128, 96, 64) == size(0, 2, 5, 128, 64, 64) == size(1, 2, 5, 0, 64, 64) == 0
    assert size(1, 1, 1, 64, 64, 64) == 0
    for Lq in (1, 32, 33, 300):
        n = size(1, 2, Lq, 9000, 64, 64)
        assert n > 0 and size(2, 2, Lq, 9000, 64, 64) >= n
        for is_dense in (False, True):
            over = dict(Lq=Lq, Lk=9000, n_table=200, ws=FAKE, ws_bytes=n - 1)
            assert _attend(lib, is_dense, **over) == S.ERR_WORKSPACE
            assert "smaller" in S.last_error()


def test_ranges_fill_the_chip(lib):
    """Cuts by the rule: none for short lists, whole work-groups over the 256 CUs for long ones."""
    cut = lib.sparstar_internal_paged_ranges
    assert cut(1, 8, 1, 1152, 64, 64, 0) == 1
    assert cut(2, 24, 1, 84_032, 128, 64, 0) == 10  # 480 work-groups of four waves, two to a CU
    assert cut(1, 1, 7, 144_512, 128, 64, 0) == 64
    assert cut(1, 24, 1, 144_512, 128, 64, 20) == 1  # short lists of a long cache
    assert cut(600, 1, 1, 144_512, 128, 64, 0) == 1
    assert cut(1, 24, 128, 144_512, 128, 64, 0) == 21  # 504 work-groups of 128 rows
    assert cut(1, 18, 220, 10_061, 128, 64, 0) == 14


# ---- the binding's own checks
def test_binding_checks_rotations():
    x, table = _t(2, 3, 9, 64), _t(20, 32, 2, dtype=F32)
    for bad in (dict(x=x.float()), dict(x=_t(3, 9, 64)), dict(x=_t(2, 3, 64, 9).transpose(2, 3)), dict(table=_t(20, 64, dtype=F32)),
                dict(table=_t(20, 32, 2)), dict(table=_t(20, 32, 3, dtype=F32)), dict(positions=_t(2, 8, dtype=I32)),
                dict(positions=_t(2, 9, dtype=torch.int64)), dict(out=_t(2, 3, 8, 64)), dict(out=_t(2, 3, 9, 64, dtype=F32))):
        a = {**dict(x=x, table=table, positions=None, out=None), **bad}
        for call in (S.sparstar_rope_fwd, S.sparstar_rope_bwd):
            with pytest.raises(ValueError):
                call(a["x"], a["table"], positions=a["positions"], out=a["out"])
    coords = _t(20, 2, dtype=I32)
    for bad in (dict(coords=coords.long().as_subclass(type(coords))), dict(coords=_t(20, dtype=I32)), dict(axis=[0]),
                dict(out=_t(20, 3, 2, dtype=F32))):
        a = {**dict(coords=coords, freq=[1.0, 0.5], axis=[0, 1], out=None), **bad}
        with pytest.raises(ValueError):
            S.sparstar_rope_table(a["coords"], a["freq"], a["axis"], out=a["out"])


def test_binding_checks_pages():
    c = S.PagedCache(_t(4, 2, 64, 32, dtype=U8), _t(4, 2, 64, 32, dtype=U8), _t(4, 2, 64, 2, dtype=U8), _t(4, 2, 64, 2, dtype=U8))
    k, q, pages = _t(1, 2, 5, 64), _t(1, 2, 8, 64), _t(1, 2, dtype=I32)
    assert c.block_size == 64
    for bad in (dict(c=c._replace(v=_t(4, 2, 64, 31, dtype=U8))), dict(c=c._replace(k=_t(4, 2, 64, 32, dtype=torch.int8))),
                dict(c=c._replace(k_scale=_t(4, 2, 64, 4, dtype=U8))), dict(c=c._replace(k=_t(2, 64, 32, dtype=U8))),
                dict(pages=_t(2, 2, dtype=I32)), dict(pages=_t(2, dtype=I32)), dict(pages=_t(1, 2, dtype=torch.int64))):
        a = {**dict(c=c, pages=pages), **bad}
        with pytest.raises(ValueError):
            S.sparstar_paged_write(k, k, a["c"], a["pages"])
        with pytest.raises(ValueError):
            S.sparstar_paged_dense_attn_fwd(q, a["c"], a["pages"])
        if a["pages"].shape[0] == 1:  # (a read takes B from the pages)
            with pytest.raises(ValueError):
                S.sparstar_paged_read(a["c"], a["pages"], 0, 5)
    for bad in (dict(v=_t(1, 2, 6, 64)), dict(starts=_t(2, dtype=I32)), dict(counts=_t(1, dtype=torch.int64)),
                dict(positions=_t(1, 4, dtype=I32)), dict(table=_t(10, 32, dtype=F32))):
        a = {**dict(v=k, starts=None, counts=None, positions=None, table=None), **bad}
        with pytest.raises(ValueError):
            S.sparstar_paged_write(k, a["v"], c, pages, starts=a["starts"], counts=a["counts"], positions=a["positions"],
                                   table=a["table"])
    for bad in (dict(lens=_t(2, dtype=I32)), dict(out=k), dict(lse=_t(1, 2, 9, dtype=F32)), dict(workspace=_t(8, 8, dtype=U8).t())):
        with pytest.raises(ValueError):
            S.sparstar_paged_dense_attn_fwd(q, c, pages, **bad)
