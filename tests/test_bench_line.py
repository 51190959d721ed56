"""The benchmark's line on stdout stays short enough to be kept whole by whoever keeps the last 3000 characters of an output."""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
import bench  # noqa: E402

PI = 3.141592653589793


def a_line():
    """Every key of the default run, with numbers of full length and texts of the longest ones' length."""
    return {"metric": bench.METRIC, "value": 1000 * PI, "unit": bench.UNIT, "n_gpus": 8, "steps": 100, "warmup": 10, "ms_per_step": PI, "higher_is_better": True,
            "scaling": "weak", "vs_baseline": None, "dtype": "f32", "data": "synthetic",
            "config": {"workload": "x" * 60, "layers": 80, "linears_per_step": 560, "batch": 1, "table_entries": "fp32, mu = 4", "Kb": 2, "Ks": 1, "salient_frac": 0.05,
                       "g": 128, "packed_bytes_resident": 10 ** 10, "algorithmic_bytes_per_step": 10 ** 10, "l2": "x" * 60, "launch": "x" * 160, "parallelism": "single GPU"},
            "us_per_layer": 10 * PI, "us_per_linear": PI, "frac_of_8TBps": PI, "step_ms_min_median_max": [PI] * 3,
            "roofline": {"bound": "hbm", "achieved": 1000 * PI, "peak": 6450.9, "unit": "GB/s", "frac": PI, "traffic": 1e10 * PI, "peak_source": "x" * 60,
                         "achieved_best_step": 1000 * PI, "frac_best_step": PI, "kernel": "x" * 24, "per": "x" * 40, "sustained": {"note": "x" * 300}},
            "e2e": {"value": 1000 * PI, "unit": bench.UNIT, "h2d_bytes_per_step": 10 ** 8, "d2h_bytes_per_step": 10 ** 8, "ms_per_step": PI, "overlap": "x" * 80,
                    "max_diff_vs_device_run": 0.0},
            "gpu_launches": 10 ** 5, "clocks": {"sm_mhz": 1965.0, "sm_max_mhz": 1965.0, "reasons": ["sw_power_cap"], "power_w": 1000.0, "samples": 100, "x": "x" * 60},
            "setup_s": 100.0, "effective_tflops": 100 * PI, "joules_per_step_lower_bound": PI, "cpu_baseline": {"x": "x" * 320}, "sections_s": 100.0,
            **{k: ["x" * 100] * 60 for k in bench.LONG}}


def test_the_line_is_short_and_nothing_is_lost():
    line = a_line()
    short, beside = bench.split_line(line)
    assert len(json.dumps(short)) < 2900
    assert {"metric", "value", "unit", "n_gpus", "steps", "warmup", "ms_per_step", "config", "e2e", "gpu_launches", "clocks", "roofline", "cpu_baseline"} <= set(short)
    assert set(beside) == {*bench.LONG, "sustained"} and beside["sustained"] == line["roofline"]["sustained"]
    assert {**short, **beside}.keys() == line.keys() | {"sustained"} and "sustained" in line["roofline"]


def test_a_line_without_sections():
    line = {k: v for k, v in a_line().items() if k not in bench.LONG}
    line["roofline"] = {k: v for k, v in line["roofline"].items() if k != "sustained"}
    assert bench.split_line(line) == (line, {})
