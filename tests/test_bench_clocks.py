"""The bench's clock sampler starts its first process before the timed region."""
import time

import bench


def test_the_first_sample_has_started_on_entry(monkeypatch):
    started = []

    class SlowPopen:
        def __init__(self, *args, **kw):
            time.sleep(0.3)
            started.append(time.perf_counter())

        def communicate(self, *args, **kw):
            return "2070, 2070, Not Active, Not Active, Not Active, Active\n", None

        def poll(self):
            return 0

        def __enter__(self):
            return self

        def __exit__(self, *exc):
            return False
        returncode = 0

    monkeypatch.setattr(bench.subprocess, "Popen", SlowPopen)
    with bench.ClockSampler(0) as clocks:
        assert started and started[0] <= time.perf_counter()
    s = clocks.summary()
    assert s["sm_mhz"] == 2070.0 and s["reasons"] == ["sw_power_cap"] and s["samples"] >= 1


def test_a_missing_tool_leaves_no_samples(monkeypatch):
    def missing(*args, **kw):
        raise FileNotFoundError("nvidia-smi")

    monkeypatch.setattr(bench.subprocess, "Popen", missing)
    with bench.ClockSampler(0) as clocks:
        pass
    assert clocks.summary() == {"sm_mhz": None, "sm_max_mhz": None, "reasons": [], "samples": 0}
