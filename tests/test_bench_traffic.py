"""The measured traffic that the benchmark reports is of the present kernels (no GPU needed)."""
import json
import os

import pytest

import bench
import synth

PROFILES = os.path.join(bench.ROOT, "profiles")
FILES = sorted(f for f in os.listdir(PROFILES) if f.startswith("traffic_") and f.endswith(".json"))


@pytest.mark.parametrize("name", FILES)
def test_kept_traffic_is_of_the_current_kernel(name):
    with open(os.path.join(PROFILES, name)) as f:
        t = json.load(f)
    assert name == f"traffic_{t['kernel_class']}_{t['workload']}.json"
    got, source = bench.measured_traffic(t["kernel_class"], t["workload"])
    assert got == t["hbm_bytes_per_launch"], source


def test_default_workload_has_one():
    workload = getattr(synth, bench.WORKLOADS["c5"]).name
    assert any(name.endswith(f"_{workload}.json") for name in FILES)
