"""The one line that bench.py prints: the contract's numbers untouched, and short enough to be read from an output's end."""
import importlib.util
import json
from pathlib import Path

from paper_2608_15473_b200 import workloads as wl

spec = importlib.util.spec_from_file_location("qf_bench", Path(__file__).resolve().parents[1] / "bench.py")
bench = importlib.util.module_from_spec(spec)
spec.loader.exec_module(bench)


def full_record():
    """A record of the shape that a default run makes, with as many repeats as there may be."""
    ms, mhz = [0.3055559992790222] * bench.MAX_REPEATS, [1875.0] * bench.MAX_REPEATS
    long = "x" * 300
    parity = {"max_abs_o_part": 1.3232299272032677e-06, "max_rel_m_part": 2.123222747092706e-07, "inf_pattern_m_part": True,
              "max_rel_lse_part": 1.4196880788203071e-07, "inf_pattern_lse_part": True, "max_abs_out": 2.9884716671452205e-07,
              "max_rel_lse": 1.3546240942055435e-07, "inf_pattern_lse": True, "tolerance": {"out_max_abs": 0.002, "lse_rel": 1e-05}, "ok": True,
              "against": long}
    clocks = {"sm_mhz": 1875.0, "sm_max_mhz": 1965.0, "reasons": ["sw_power_cap", "hw_thermal_slowdown"], "samples": 195, "power_w_max": 555.622, "source": "nvml"}
    cpu = {"value": 10.706066020044391, "unit": "GB/s", "cores": 16, "kind": "oracle", "seconds": 0.18840096000002404,
           "sample": "the whole workload once: 32 requests, 491116 cached tokens, partials + combine", "single_thread": {"sample": long}}
    roof = {"bound": "hbm", "kernel": "sweep_kernel", "achieved": 6646.8423789471135, "peak": 6535.7, "unit": "GB/s", "frac": 1.017005428484648,
            "peak_kind": "of measured", "frac_of_datasheet_8TBs": 0.8308552973683891, "ms_per_launch": 0.3030399978160858,
            "bytes_per_launch": 2014259100, "traffic": 2019076744, "note": long, "min_ms_per_launch": 0.30105599761009216}
    args = type("A", (), dict(workload=3, seed=0, kv_layout="hnd"))
    rec = {"metric": bench.METRIC, "value": 6601.189702572724, "unit": "GB/s", "n_gpus": 1, "steps": 20, "warmup": 5, "ms_per_step": 0.3055559992790222,
           "higher_is_better": True, "scaling": "weak", "vs_baseline": None, "dtype": "bf16", "data": "synthetic",
           "config": bench.config_record(args, wl.CONFIGS[1](seed=0), 1), "timing": bench.spread(ms, mhz), "clocks": clocks,
           "e2e": {"value": 6574.524172961269, "unit": "GB/s", "h2d_bytes_per_step": 264704, "d2h_bytes_per_step": 528384,
                   "ms_per_step": 0.30679529999986244, "min_ms_per_step": 0.3062578500021118, "max_ms_per_step": 0.3070745000002262,
                   "synchronous_ms_per_step": 0.3502324500004761, "synchronous_min_ms": 0.34972994999975526, "note": long},
           "gpu_launches": 60, "roofline": roof, "kv_tokens_per_s": 1607286393.1941044, "pct_of_hbm_peak": 82.51487128215905,
           "pct_of_measured_copy": 101.00203042631583, "sweep_kernel_pct_of_hbm_peak": 83.08552973683892, "parity": parity, "cpu_baseline": cpu}
    names = [bench.workload_name(4), bench.workload_name(4) + " (shuffled table)", bench.workload_name(2), bench.workload_name(5),
             bench.workload_name(3) + " (token-major pages [page, 16, Hkv, D])", bench.workload_name(1)]
    rec["also"] = [{"workload": n, "ms_per_step": 0.6028783798217774, "GB/s": 7124.9975978071, "timing": rec["timing"], "parity": parity} for n in names]
    rec["also"][3] = {"workload": names[3], "error": "RuntimeError: " + long}
    return rec


def test_the_line_fits_a_reader_of_the_last_3000_characters(capsys, tmp_path):
    """The whole record is 20,000 characters: a reader that keeps an output's end saw no line at all."""
    rec = full_record()
    bench.emit(rec, str(tmp_path / "record.json"))
    got = capsys.readouterr()
    assert got.out.count("\n") == 1 and len(got.out) <= bench.LINE_CHARS and got.err == ""
    assert json.loads((tmp_path / "record.json").read_text()) == rec
    line = json.loads(got.out)
    for k in ("metric", "value", "unit", "n_gpus", "steps", "warmup", "ms_per_step", "higher_is_better", "scaling", "vs_baseline", "dtype", "data",
              "config", "gpu_launches"):
        assert line[k] == rec[k], k
    assert all(line["e2e"][k] == rec["e2e"][k] for k in ("value", "unit", "h2d_bytes_per_step", "d2h_bytes_per_step"))
    assert all(line["clocks"][k] == rec["clocks"][k] for k in ("sm_mhz", "sm_max_mhz", "reasons"))
    assert [a["workload"] for a in line["also"]] == ["cfg4", "cfg4 shuffled table", "cfg2", "cfg5", "cfg3 token-major", "cfg1"]
    assert line["also"][0]["parity_ok"] is True and "RuntimeError" in line["also"][3]["error"]
    assert abs(line["roofline"]["frac"] / rec["roofline"]["frac"] - 1) < 1e-5


def test_the_line_of_a_record_without_the_optional_parts():
    rec = {k: v for k, v in full_record().items() if k not in ("also", "e2e", "parity", "cpu_baseline", "roofline")}
    assert bench.short_line(rec)["value"] == rec["value"] and "also" not in bench.short_line(rec)
