"""Which sources the bench's measured HBM traffic belongs to."""
import os
import re
import shutil

import pytest

import bench

CSRC = os.path.join(bench.ROOT, "paper_2103_00686_amd", "csrc")


def _text(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


@pytest.mark.parametrize("kernel", sorted(bench.KERNEL_CLASS))
def test_every_measured_kernel_s_source_counts(kernel):
    at = [n for n in os.listdir(CSRC) if n.endswith((".hip", ".h")) and re.search(rf"__global__[^;{{]*\b{kernel}\(", _text(n))]
    assert at and set(at) <= set(bench.TRAFFIC_SOURCES)


def test_and_what_these_include():
    for name in bench.TRAFFIC_SOURCES:
        assert set(re.findall(r'#include "(fae_\w+\.h)"', _text(name))) <= set(bench.TRAFFIC_SOURCES)


def test_other_kernels_leave_the_figures(tmp_path, monkeypatch):
    """A new source, or a changed one of other kernels, is not a reason to drop them; a changed one of theirs is."""
    to = tmp_path / "paper_2103_00686_amd" / "csrc"
    shutil.copytree(CSRC, to)
    here = bench.csrc_hash()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.csrc_hash() == here
    (to / "fae_of_its_own.hip").write_text("// another kernel\n")
    (to / "fae_dropout.hip").write_text("// changed\n")
    assert bench.csrc_hash() == here
    with open(to / "fae_bwd_reduce.hip", "a") as f:
        f.write("// changed\n")
    assert bench.csrc_hash() != here
