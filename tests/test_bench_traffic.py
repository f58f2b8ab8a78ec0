"""bench.py reports counted traffic only for the sources that it was counted with."""
import os
import shutil

import pytest

import bench

FILES = ["cp_extend.hip", "cp_decode.h", "cp_device.h"]     # the kernels' device code


@pytest.fixture()
def copied(tmp_path, monkeypatch):
    folder = os.path.join("paper_2511_03475_amd", "csrc")
    shutil.copytree(os.path.join(bench.ROOT, folder), tmp_path / folder)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    monkeypatch.setitem(bench.TRAFFIC, "source_sha256_16", bench.source_digest())
    return tmp_path / folder


def test_the_same_sources_have_their_traffic(copied):
    for workload in ("long_context_32k", "decode_b32_p10k"):
        assert bench.measured_traffic(workload) == bench.TRAFFIC[workload]
    (copied / "cp_pages.hip").write_text("// a file that they do not include\n")
    assert bench.measured_traffic("decode_b32_p10k") is not None


@pytest.mark.parametrize("name", FILES)
def test_a_change_of_any_file_of_the_kernels_takes_it_away(copied, name):
    with open(copied / name, "a") as f:
        f.write("// changed\n")
    assert bench.measured_traffic("long_context_32k") is None and bench.measured_traffic("decode_b32_p10k") is None


def test_missing_sources_have_none(copied):
    (copied / "cp_decode.h").unlink()
    assert bench.measured_traffic("decode_b32_p10k") is None
