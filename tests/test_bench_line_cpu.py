"""The benchmark's line stays short: its long sections are a record of their own."""
import json


def test_long_sections_leave_the_line():
    import bench
    line = {"metric": bench.METRIC, "value": 1.0, "unit": bench.UNIT, "e2e": {"value": 2.0}, "clocks": {"sm_mhz": 1.0},
            "decode": {"decode_us_per_layer_step": 3.0, "append": {"us": 4.0}, "configs": [{"x": "y" * 100}] * 90},
            "sweep": [{"x": "y" * 200}] * 48, "decode_summary": {"cfg1": [1, 2]}}
    kept = json.dumps(line)
    short, details = bench.split_details(line)
    assert json.dumps(line) == kept                                    # the caller's object is left alone
    assert len(json.dumps(short)) < 1000
    assert short["decode"] == {"decode_us_per_layer_step": 3.0, "append": {"us": 4.0}}
    assert {k: v for k, v in short.items() if k != "decode"} == {k: v for k, v in line.items() if k not in ("decode", "sweep")}
    assert details == {"sweep": line["sweep"], "decode": {"configs": line["decode"]["configs"]}}
    assert bench.split_details({"metric": 1}) == ({"metric": 1}, {"sweep": None})
