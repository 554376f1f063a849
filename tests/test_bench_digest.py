"""What makes the recorded DRAM counters stale, on CPU with a copy of the sources."""
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import bench  # noqa: E402

CSRC = os.path.join("paper_2004_14180_b200", "csrc")


@pytest.fixture
def csrc(tmp_path, monkeypatch):
    shutil.copytree(os.path.join(ROOT, CSRC), tmp_path / CSRC)
    before = bench.csrc_digest()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.csrc_digest() == before
    return tmp_path / CSRC, before


@pytest.mark.parametrize("name", ["qadam_api.cu", "qadam_host.h", "qadam_device.cuh", "qadam_kernels.cuh", "qadam_noalloc.cu",
                                  "qadam_server_pipe.cuh", "qadam_worker_resident.cuh", "qadam_worker_stream.cuh", "a_new_header.cuh"])
def test_a_change_of_the_step_makes_the_counters_stale(csrc, name):
    base, before = csrc
    with open(base / name, "a") as f:
        f.write("\n")
    assert bench.csrc_digest() != before


def test_a_change_of_other_operators_does_not(csrc):
    base, before = csrc
    for name in bench.OTHER_OPERATORS:
        with open(base / name, "a") as f:
            f.write("\n")
    assert bench.csrc_digest() == before
