"""Reads of the paged cache whose work-groups do not fill their grid: the work of each on the CPU
(tests/asan/read_groups.cpp), and such a read on the GPU."""
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_piece_is_read_once_and_nothing_else(tmp_path):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the ROCm headers are not available")
    exe = str(tmp_path / "read_groups")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "asan", "read_groups.cpp"), "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True)
    assert b.returncode == 0, b.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]


@pytest.mark.gpu
@pytest.mark.parametrize("want", ["k", "v"])
@pytest.mark.parametrize("D,L", [(128, (1 << 25) + 1), (64, (1 << 26) + 1)])
def test_a_read_of_one_half_past_a_row_of_work_groups(gpu_lib, D, L, want):
    """2^20 + 1 work-groups, in two rows of 524,289: one too many."""
    S, block, n = gpu_lib, 64, 4
    print(f"[paged read] {want} alone, D={D}, {L} rows", flush=True)
    g = torch.Generator().manual_seed(D)
    c = S.PagedCache.empty(n, 1, D, block)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        scale.copy_(torch.randint(122, 128, scale.shape, generator=g, dtype=torch.uint8))
    few = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    period = n * block
    ref = S.sparstar_paged_read(c, few, 0, period)["kv".index(want)].view(period, D)
    pages = few.repeat(1, -(-L // period))
    whole = torch.full((L + 64, D), 9.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:L].view(1, 1, L, D)
    S.sparstar_paged_read(c, pages, 0, L, out=(out, None) if want == "k" else (None, out))
    torch.cuda.synchronize()
    assert (whole[L:] == 9).all() and torch.equal(whole[L - 1], ref[(L - 1) % period])
    rows = out.view(L, D)[: L - 1].view(-1, period, D)
    for at in range(0, rows.shape[0], 1 << 14):
        assert (rows[at: at + (1 << 14)] == ref).all()
