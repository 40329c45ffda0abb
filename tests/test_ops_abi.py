"""Refusals of the gradient and cache entry points, and the cuts their plans make: on the
host, without a GPU (the fake device pointers are never dereferenced)."""
import ctypes
import os

import pytest
import torch

from paper_2608_10519_amd import sparstar as S

FAKE = 0x10000
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.fail("libsparstar.so is not built (run __graft_entry__.build())")
    return S.load()


def _bwd(lib, dense=False, **over):
    a = dict(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, d_o=FAKE, d_lse=None, B=1, H=2, Lq=512, Lk=1152, D=64, block=64,
             num=FAKE, idx=FAKE, stride=6, scale=0.0, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(over)
    head = [a[x] for x in ("q", "k", "v", "o", "lse", "d_o", "d_lse", "B", "H", "Lq", "Lk", "D", "block")]
    tail = [a[x] for x in ("scale", "dq", "dk", "dv", "ws", "ws_bytes")] + [None]
    if dense:
        return lib.sparstar_dense_attn_bwd(*head, *tail)
    return lib.sparstar_sparse_attn_bwd(*head, a["num"], a["idx"], a["stride"], *tail)


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("over,code,msg", [
    (dict(D=96), S.ERR_UNSUPPORTED, "head dim"),
    (dict(block=32), S.ERR_UNSUPPORTED, "block size"),
    (dict(B=0), S.ERR_INVALID_ARG, "B and H"),
    (dict(Lk=0), S.ERR_INVALID_ARG, "Lk"),
    (dict(Lq=-1), S.ERR_INVALID_ARG, "Lq"),
    (dict(q=None), S.ERR_INVALID_ARG, "non-null"),
    (dict(lse=None), S.ERR_INVALID_ARG, "non-null"),
    (dict(d_o=None), S.ERR_INVALID_ARG, "non-null"),
    (dict(dv=None), S.ERR_INVALID_ARG, "non-null"),
    (dict(o=FAKE + 8), S.ERR_INVALID_ARG, "16-byte"),
    (dict(dk=FAKE + 2), S.ERR_INVALID_ARG, "16-byte"),
    (dict(lse=FAKE + 2), S.ERR_INVALID_ARG, "4-byte"),
    (dict(d_lse=FAKE + 1), S.ERR_INVALID_ARG, "4-byte"),
    (dict(scale=float("nan")), S.ERR_INVALID_ARG, "finite"),
    (dict(scale=float("inf")), S.ERR_INVALID_ARG, "finite"),
    (dict(ws=None), S.ERR_WORKSPACE, "null"),
    (dict(ws=FAKE + 16), S.ERR_WORKSPACE, "256-byte"),
    (dict(ws_bytes=100), S.ERR_WORKSPACE, "smaller"),
])
def test_gradients_refuse(lib, dense, over, code, msg):
    assert _bwd(lib, dense, **over) == code
    assert msg in S.last_error()


@pytest.mark.parametrize("over,msg", [(dict(num=None), "kv_num_blocks"), (dict(idx=None), "kv_indices"),
                                      (dict(stride=0), "kv_stride")])
def test_sparse_gradient_refuses_lists(lib, over, msg):
    assert _bwd(lib, **over) == S.ERR_INVALID_ARG
    assert msg in S.last_error()


def test_gradient_workspace_is_enough_for_both_calls(lib):
    n = S.sparstar_attn_bwd_workspace_bytes(1, 2, 512, 1152, 64, 64)
    assert n > 0
    for dense in (False, True):
        assert _bwd(lib, dense, ws_bytes=255) == S.ERR_WORKSPACE
    assert S.sparstar_attn_bwd_workspace_bytes(1, 2, 512, 1152, 96, 64) == 0
    assert S.sparstar_attn_bwd_workspace_bytes(0, 2, 512, 1152, 64, 64) == 0


def bwd_plan(lib, B, H, Lq, Lk, D, block, dense):
    out = (ctypes.c_int64 * 2)()
    i64 = ctypes.c_int64
    lib.sparstar_internal_bwd_plan(B, H, i64(Lq), i64(Lk), D, block, int(dense), out)
    return tuple(out)


def cache_plan(lib, B, H, Lq, Lk, D, block, kv_stride=0):
    out = (ctypes.c_int64 * 2)()
    i64 = ctypes.c_int64
    lib.sparstar_internal_cache_plan(B, H, i64(Lq), i64(Lk), D, block, i64(kv_stride), out)
    return tuple(out)


def test_plans_cut_where_work_groups_are_few(lib):
    assert bwd_plan(lib, 1, 24, 72_000, 144_512, 128, 64, False) == (1, 1)
    dq, dkv = bwd_plan(lib, 1, 1, 64, 8192, 128, 64, False)
    assert dq > 1 and dkv == 1
    dq, dkv = bwd_plan(lib, 1, 1, 8192, 64, 128, 64, True)
    assert dq == 1 and dkv > 1
    assert cache_plan(lib, 1, 1, 1, 64, 128, 64) == (1, 1)
    waves, ranges = cache_plan(lib, 2, 24, 1, 84_032, 128, 64)
    assert waves == 1 and ranges > 8


def _write(lib, **over):
    a = dict(k=FAKE, v=FAKE, B=1, H=2, L=5, D=64, block=64, start=3, starts=None, counts=None, cap=128, kc=FAKE, vc=FAKE,
             ks=FAKE, vs=FAKE)
    a.update(over)
    return lib.sparstar_cache_write(*[a[x] for x in ("k", "v", "B", "H", "L", "D", "block", "start", "starts", "counts",
                                                     "cap", "kc", "vc", "ks", "vs")], None)


@pytest.mark.parametrize("over,msg", [
    (dict(D=96), "head dim"), (dict(block=32), "block size"), (dict(H=0), "B and H"), (dict(L=-1), "Lq"),
    (dict(cap=0), "capacity"), (dict(cap=(1 << 30) + 1), "capacity"), (dict(start=-1), "inside"),
    (dict(start=124), "inside"), (dict(start=129, L=0), "inside"), (dict(k=None), "non-null"),
    (dict(kc=None), "four arrays"), (dict(vs=None), "four arrays"), (dict(v=FAKE + 2), "16-byte"),
    (dict(vc=FAKE + 8), "16-byte"), (dict(starts=FAKE + 2), "4-byte"),
])
def test_cache_write_refuses(lib, over, msg):
    assert _write(lib, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
    assert msg in S.last_error()


def test_cache_write_of_nothing(lib):
    assert _write(lib, L=0) == S.OK
    assert _write(lib, L=0, start=128, k=None, v=None) == S.OK


def _read(lib, **over):
    a = dict(kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, B=1, H=2, start=3, L=5, cap=128, D=64, block=64, k=FAKE, v=FAKE)
    a.update(over)
    return lib.sparstar_cache_read(*[a[x] for x in ("kc", "vc", "ks", "vs", "B", "H", "start", "L", "cap", "D", "block",
                                                    "k", "v")], None)


@pytest.mark.parametrize("over,msg", [
    (dict(D=32), "head dim"), (dict(start=124), "inside"), (dict(start=-1), "inside"), (dict(ks=None), "four arrays"),
    (dict(k=FAKE + 8), "16-byte"),
])
def test_cache_read_refuses(lib, over, msg):
    assert _read(lib, **over) in (S.ERR_INVALID_ARG, S.ERR_UNSUPPORTED)
    assert msg in S.last_error()


def test_cache_read_of_nothing(lib):
    assert _read(lib, L=0) == S.OK
    assert _read(lib, k=None, v=None) == S.OK


def _attend(lib, dense=False, **over):
    a = dict(q=FAKE, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, B=1, H=2, Lq=512, Lk=1152, cap=1200, D=64, block=64, lens=None,
             num=FAKE, idx=FAKE, stride=6, scale=0.0, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(over)
    head = [a[x] for x in ("q", "kc", "vc", "ks", "vs", "B", "H", "Lq", "Lk", "cap", "D", "block", "lens")]
    tail = [a[x] for x in ("scale", "o", "lse", "ws", "ws_bytes")] + [None]
    if dense:
        return lib.sparstar_cache_dense_attn_fwd(*head, *tail)
    return lib.sparstar_cache_sparse_attn_fwd(*head, a["num"], a["idx"], a["stride"], *tail)


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("over,code,msg", [
    (dict(D=96), S.ERR_UNSUPPORTED, "head dim"),
    (dict(block=96), S.ERR_UNSUPPORTED, "block size"),
    (dict(Lk=0), S.ERR_INVALID_ARG, "Lk"),
    (dict(Lk=1201), S.ERR_INVALID_ARG, "exceeds"),
    (dict(cap=0), S.ERR_INVALID_ARG, "capacity"),
    (dict(q=None), S.ERR_INVALID_ARG, "q and o"),
    (dict(o=FAKE + 4), S.ERR_INVALID_ARG, "16-byte"),
    (dict(kc=FAKE + 4), S.ERR_INVALID_ARG, "16-byte"),
    (dict(lens=FAKE + 2), S.ERR_INVALID_ARG, "4-byte"),
    (dict(vs=None), S.ERR_INVALID_ARG, "four arrays"),
    (dict(scale=float("nan")), S.ERR_INVALID_ARG, "finite"),
    (dict(ws=FAKE + 16), S.ERR_WORKSPACE, "256-byte"),
    (dict(Lq=1, Lk=1152, ws_bytes=16, stride=18), S.ERR_WORKSPACE, "smaller"),
])
def test_cache_attention_refuses(lib, dense, over, code, msg):
    assert _attend(lib, dense, **over) == code
    assert msg in S.last_error()


@pytest.mark.parametrize("over,msg", [(dict(num=None), "kv_num_blocks"), (dict(stride=0), "kv_stride")])
def test_sparse_cache_attention_refuses_lists(lib, over, msg):
    assert _attend(lib, **over) == S.ERR_INVALID_ARG
    assert msg in S.last_error()


def test_cache_attention_without_queries(lib):
    assert _attend(lib, Lq=0, q=None, o=None) == S.OK


def test_binding_refuses_before_the_library():
    t = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)  # not on the GPU
    with pytest.raises(ValueError):
        S.sparstar_dense_attn_bwd(t, t, t, t, torch.zeros(1, 1, 4), t)
    c = S.KvCache.empty(1, 1, 64, 64, 64, device="cpu")
    assert c.k.shape == (1, 1, 64, 64) and c.k_scale.shape == (1, 1, 1)
    with pytest.raises(ValueError):
        S.sparstar_cache_write(t, t, c)
    with pytest.raises(ValueError):
        S.sparstar_cache_dense_attn_fwd(t, c)
    with pytest.raises(ValueError):
        S.sparstar_cache_read(c, 0, 4)
