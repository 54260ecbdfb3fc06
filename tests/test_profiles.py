"""The figures that bench.py takes from profiles/ are those of the trace document beside them, with its stamp."""
import json
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_traffic_is_what_the_trace_document_says():
    with open(os.path.join(ROOT, "profiles", "traffic_cfg2_qwen1.5b.json")) as f:
        traffic = json.load(f)
    with open(os.path.join(ROOT, "profiles", "bench_cfg2_qwen1.5b_kernel_trace_and_traffic.md")) as f:
        text = f.read()
    assert re.findall(r"`rapid_version\(\)` = (\d+)", text) == [str(traffic["rapid_version"])]
    fetch, write = (float(x) for x in re.search(r"\(mean ([0-9.]+)\), WRITE_SIZE .*?\(mean ([0-9.]+)\)", text).groups())
    rows = 0
    for mode, part in zip(re.findall(r"^# Mode `(\w+)`", text, flags=re.M), re.split(r"^# Mode `\w+`", text, flags=re.M)[1:]):
        for e in traffic["modes"][mode].values():
            kib = re.search(r"^\| " + re.escape(e["kernel"]) + r" \| " + str(e["rows_per_launch"]) + r" \| ([0-9.e+]+) \| ([0-9.e+]+) \|", part, flags=re.M)
            # four digits each of the counters, three of the factors
            assert abs(float(kib[1]) * 1024 / fetch / e["read_bytes"] - 1) < 2e-3 and abs(float(kib[2]) * 1024 / write / e["written_bytes"] - 1) < 2e-3
            assert e["bytes_per_launch"] == e["read_bytes"] + e["written_bytes"]
            rows += 1
    assert rows == sum(len(m) for m in traffic["modes"].values()) == 10
