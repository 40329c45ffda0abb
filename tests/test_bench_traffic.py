"""bench.py reports the attention kernel's measured HBM traffic only while every source that the
measurement depends on is what it was."""
from __future__ import annotations

import shutil

import pytest

import bench


@pytest.fixture
def copied(tmp_path, monkeypatch):
    """The sources in a folder of their own, and a summary measured on them."""
    shutil.copytree(bench.CSRC, tmp_path / "csrc")
    monkeypatch.setattr(bench, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(bench, "TRAFFIC_SUMMARY", str(tmp_path / "hbm.md"))
    (tmp_path / "hbm.md").write_text(f"kernel_source_sha256: {bench.attention_source_hash()}\n"
                                     "fetch_bytes_per_launch: 1.5e+11\nwrite_bytes_per_launch: 2e+09\n")
    return tmp_path


def test_traffic_of_the_measured_sources(copied):
    assert bench.traffic_from_profile() == {"fetch": 1.5e11, "write": 2e9}
    (copied / "hbm.md").unlink()
    assert bench.traffic_from_profile() is None


@pytest.mark.parametrize("name", ["attn_fwd.hip", "attn_device.h", "device_common.h", "launch.h", "attn_plan.h"])
def test_no_traffic_of_other_sources(copied, name):
    with open(copied / "csrc" / name, "a") as f:
        f.write("\n")
    assert bench.traffic_from_profile() is None
    assert name in bench.attention_sources()


def test_sources_of_other_kernels_do_not_matter(copied):
    with open(copied / "csrc" / "cache_attn.hip", "a") as f:
        f.write("\n")
    assert bench.traffic_from_profile() is not None
