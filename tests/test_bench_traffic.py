"""bench.py reports recorded DRAM traffic only for the kernel sources that it was measured on."""
import os
import re
import shutil

import pytest

import bench

CSRC = os.path.join(bench.ROOT, "paper_2503_21817_b200", "csrc")


def test_recorded_traffic_of_the_sources_it_was_measured_on(monkeypatch):
    monkeypatch.setattr(bench, "NCU_TRAFFIC_SOURCE_SHA", bench.ncu_traffic_source_sha(CSRC))
    assert bench.ncu_traffic("gateup") == bench.NCU_TRAFFIC_BYTES["gateup"]
    assert bench.ncu_traffic("no such kernel") is None
    assert bench.ncu_traffic("gateup", os.path.join(bench.ROOT, "tests")) is None


def test_every_header_of_the_measured_kernels_counts():
    for name in bench.NCU_TRAFFIC_SOURCES:
        for header in re.findall(r'#include "(\w+\.cuh)"', open(os.path.join(CSRC, name)).read()):
            assert header in bench.NCU_TRAFFIC_SOURCES, (name, header)


@pytest.mark.parametrize("name", bench.NCU_TRAFFIC_SOURCES)
def test_a_change_to_any_of_them_voids_it(name, tmp_path, monkeypatch):
    for n in bench.NCU_TRAFFIC_SOURCES:
        shutil.copy(os.path.join(CSRC, n), tmp_path / n)
    monkeypatch.setattr(bench, "NCU_TRAFFIC_SOURCE_SHA", bench.ncu_traffic_source_sha(str(tmp_path)))
    assert bench.ncu_traffic("gateup", str(tmp_path)) is not None
    with open(tmp_path / name, "a") as f:
        f.write("// changed\n")
    assert bench.ncu_traffic("gateup", str(tmp_path)) is None
