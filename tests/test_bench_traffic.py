"""DRAM traffic that the benchmark takes from recorded captures: only for kernels whose sources are those that were captured."""
import json
import os
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2405_18428_b200", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC)
    shutil.copytree(os.path.join(bench.ROOT, "profiles"), tmp_path / "profiles")
    record = tmp_path / "profiles" / "dram_traffic.json"
    rec = json.loads(record.read_text())
    # as if all had been captured with the sources that are there
    rec["sources"] = {f: bench.source_hash(f) for f in rec["sources"]}
    record.write_text(json.dumps(rec))
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def touched(path):
    path.write_text(path.read_text() + "\n// changed\n")


def test_each_record_names_a_source():
    with open(os.path.join(bench.ROOT, "profiles", "dram_traffic.json")) as f:
        rec = json.load(f)
    assert {k["source"] for k in rec["kernels"]} == set(rec["sources"])
    assert all(os.path.exists(os.path.join(bench.ROOT, CSRC, f)) for f in rec["sources"])


def test_a_kernel_is_recorded_until_its_own_sources_change(tree):
    ask = lambda: [bench.recorded_traffic(k, "C5") is not None for k in ("sweep_fwd", "gate_logsigmoid", "srem_dwconv3x3")]
    assert ask() == [True, True, True]
    touched(tree / "rope.cu")                # another kernel's file
    touched(tree / "decay.cuh")
    assert ask() == [True, True, True]
    touched(tree / "gate.cu")
    assert ask() == [True, False, True]
    touched(tree / "sweep_plan.cuh")         # a header of the sweeps
    assert ask() == [False, False, True]
    touched(tree / "dig_common.cuh")         # ... of all
    assert ask() == [False, False, False]
    assert bench.recorded_traffic("sweep_fwd", "C1") is None and bench.recorded_traffic("decay_pass", "C5") is None
