"""The benchmark's JSON line: short enough to be kept whole by whoever records
the last 16,000 characters of the output."""

import json

import bench


def test_legs_fit_the_line():
    leg = {"workload": "16k", "mode": "accumulate", "tau": 0.9, "late_kernel": "sparse_attn_grouped_kernel", "density": 1 / 3,
           "shape": "batch 1, 32 heads, d 128, seq 32768, block 128, 8 discovery + 24 late steps", "nnz": 938667,
           "late_ms": 10 / 3, "late_ms_iqr": [1 / 3] * 2, "late_tflops": 1e4 / 7, "dense_ms": 1 / 7, "dense_tflops": 1e4 / 7,
           "select_ms": 1 / 7, "discovery_ms": 1e3 / 7, "speedup_prepared": 8 / 7, "speedup_trajectory": 8 / 7,
           "speedup_matched_backend": 8 / 7, "retained_future_mass_mean": 1 / 7, "j_roll_mean_late": 1 / 7,
           "manifest": {"inputs_sha256": {f"step{i}": "0" * 64 for i in range(6)}}}
    brief = bench.rounded(leg)
    assert "manifest" not in brief and brief["late_ms"] == 3.33333 and brief["tau"] == 0.9
    assert len(json.dumps({f"leg{i}": brief for i in range(20)})) < 12000
