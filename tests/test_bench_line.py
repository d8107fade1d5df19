"""The line that bench.py prints: short enough to survive whoever keeps only the end of the output, with the contract's keys."""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import bench  # noqa: E402


def record():
    many = {f"workload {i}": {"tokens_per_s": 1.0 / 3.0, "clocks": {"samples": list(range(50))}} for i in range(20)}
    return {"metric": bench.METRIC, "value": 1428900.369121544, "unit": bench.UNIT, "n_gpus": 1, "steps": 20, "warmup": 5,
            "ms_per_step": 22.93231964111328, "mean_ms_per_step": 22.99954833984375, "higher_is_better": True, "scaling": "weak",
            "vs_baseline": None, "dtype": "mxfp8 routed experts (fp32 accumulate), bf16 elsewhere", "data": "synthetic",
            "config": {"workload": "deepseek_v3", "T": 32768, "H": 7168, "E": 256, "k": 8, "I": 2048, "I_shared": 2048, "routing": "none",
                       "parallelism": "token-sharded replicas x1", "h_ring_tiles": 0, "workspace_bytes": 11452540160, "l2": "x" * 75,
                       "timing": "x" * 170},
            "tflops": 1132.722838889706, "gpu_launches": 200, "per_config": many, "sweep": [many] * 3, "inputs": {"x": "y" * 200},
            "roofline": {"kernel": "k" * 150, "bound": "tensor", "achieved": 1191.771554761272, "peak": 1404.8, "unit": "TFLOP/s",
                         "frac": 0.848356744562409, "traffic_source": "t" * 100, "sustained_run": many},
            "clocks": {"sm_mhz": 1387.0, "sm_min_mhz": 1357.0, "sm_max_mhz": 1965.0, "power_w_max": 419.78, "samples": 5,
                       "reasons": ["sw_power_cap"]},
            "e2e": {"value": 1340647.684782144, "unit": "tokens/s", "ms_per_step": 24.441917419433594, "steps": 10,
                    "h2d_bytes_per_step": 469762048, "d2h_bytes_per_step": 469762048, "mode": "m" * 130, "single_call_ms": 34.417195638020836,
                    "result_bits_equal_device_call": True},
            "cpu_baseline": {"value": 68.36181663912903, "unit": "tokens/s", "cores": 16, "kind": "oracle", "sample": "s" * 100}}


def test_the_line_is_short_and_the_record_is_whole(capsys):
    full = record()
    bench.emit(full)
    out, err = capsys.readouterr()
    assert out.count("\n") == 1 and len(out) < 2000
    line = json.loads(out)
    for key in ("metric", "value", "unit", "n_gpus", "steps", "warmup", "ms_per_step", "higher_is_better", "scaling", "vs_baseline", "dtype",
                "data", "config", "clocks", "e2e", "gpu_launches"):
        assert line[key] == full[key], key
    assert line["roofline"]["frac"] == full["roofline"]["frac"] and line["cpu_baseline"]["kind"] == "oracle"
    assert json.loads(err) == full
