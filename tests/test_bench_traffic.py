"""bench.py's traffic fields: counters are reported for the kernel sources that
they were taken of, and other sources have no part in that."""
import json
import os

import pytest

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TRAFFIC = json.load(open(os.path.join(ROOT, "profiles", "traffic.json")))


def test_sources_of_a_step():
    names = {os.path.basename(f) for f in bench.kernel_sources()}
    assert {"decode.hip", "prefill.hip", "phi.hip", "glide_api.hip", "glide_internal.h", "flush.h"} <= names
    assert not any(n.startswith(("paged", "evict")) for n in names)


@pytest.mark.parametrize("name", sorted(TRAFFIC["workloads"]))
def test_counted_workloads_report_traffic(name):
    w = TRAFFIC["workloads"][name]
    assert bench.measured_traffic(name) == {"decode_step_bytes": round(w["decode_step_bytes"]),
                                            "prefill_call_bytes": round(w["prefill_call_bytes"])}


def test_changed_sources_report_none(monkeypatch, tmp_path):
    f = tmp_path / "decode.hip"
    f.write_text("changed")
    real = bench.kernel_sources()
    monkeypatch.setattr(bench, "kernel_sources", lambda: real[1:] + [str(f)])
    assert bench.measured_traffic(next(iter(TRAFFIC["workloads"]))) is None


def test_uncounted_workload_reports_none():
    assert bench.measured_traffic("no such workload") is None
