"""bench.py reports the HBM bytes that were counted for the kernels in the tree, and none for kernels that have changed since."""
import json
import os

import bench


def test_the_counted_traffic_is_of_the_kernels_in_the_tree():
    with open(os.path.join(bench.ROOT, "profiles", "traffic.json")) as f:
        counted = json.load(f)
    for name, entry in counted["kernels"].items():
        assert bench.load_traffic(name) == entry["hbm_bytes_per_launch"], name


def test_other_sources_have_no_counted_traffic(monkeypatch):
    monkeypatch.setattr(bench, "source_digest", lambda: "0" * 64)
    assert bench.load_traffic("gemm_gateup_skinny") is None
