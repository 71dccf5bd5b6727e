"""The traffic figure that the step benchmark reports goes with one capture and the sources it was taken from."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_reported_traffic_is_the_recorded_capture():
    import bench
    text = open(os.path.join(ROOT, "profiles", "attn_tc_kernel_c3_layer.md")).read()
    text = text[text.index("The traffic figure `bench.py` reports"):]
    assert bench.NCU_TRAFFIC["sha256"][:16] in text           # the capture's own sources: a digest of its own needs a capture of its own
    launches = re.findall(r"^\| \d+ \| ([\d.]+) MB \| ([\d.]+) MB \|", text, re.M)
    assert len(launches) >= 2
    mean = sum(float(r) + float(w) for r, w in launches) / len(launches)
    assert abs(mean * 1e6 - bench.NCU_TRAFFIC["bytes_per_launch"]) <= 0.06e6


def test_no_figure_for_other_sources(monkeypatch):
    import bench
    from paper_2404_12022_b200 import workloads as wl
    w = wl.config_c3()
    monkeypatch.setattr(bench, "traffic_digest", lambda: bench.NCU_TRAFFIC["sha256"])
    assert bench.ncu_traffic(w) == bench.NCU_TRAFFIC["bytes_per_launch"]
    monkeypatch.setattr(bench, "traffic_digest", lambda: "0" * 64)
    assert bench.ncu_traffic(w) is None
