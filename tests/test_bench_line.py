"""The benchmark's JSON line: one line on stdout that stays short, the records of every configuration on stderr."""
import json

import bench


def record(name):
    return dict(workload=name, ms_per_step=0.02061353830190805, value=79.76152099262896, unit="TOPS", io="fp32", variant="i8", launches_per_step=1,
                l2="9 rotating input/output sets (330 MiB) > L2", images_per_s=12345.678901,
                roofline=dict(bound="hbm", achieved=1869.8080569909878, peak=6551.7, unit="GB/s", frac=0.2853928075142311, peak_source="s" * 100),
                e2e=dict(value=1.5711357047467844, unit="TOPS", h2d_bytes_per_step=51380224, d2h_bytes_per_step=25690112, overlap="s" * 80),
                timing=dict(regions=5, region_ms=[48.219] * 5, statistic="median over regions"),
                clocks=dict(sm_mhz=1965.0, sm_max_mhz=1965.0, samples=12, reasons=["sw_power_cap"], window="s" * 80))


def test_the_line_is_short_and_the_records_whole(capsys):
    entries = [record(n) for n in bench.SUITE]
    head = dict(metric=bench.METRIC, value=1.0, peaks="p" * 1200, config="c" * 800, roofline="r" * 600)
    bench.report(head, entries)
    out = capsys.readouterr()
    lines = out.out.splitlines()
    assert len(lines) == 1 and len(lines[0]) < 8000
    got = json.loads(lines[0])
    assert [e["workload"] for e in got["per_config"]] == list(bench.SUITE)
    assert got["per_config"][0] == dict(workload=bench.SUITE[0], ms_per_step=0.0206135, value=79.7615, unit="TOPS", images_per_s=12345.7, launches_per_step=1,
                                        bound="hbm", frac=0.285393, e2e=1.57114, sm_mhz=1965.0, reasons=["sw_power_cap"])
    records = [json.loads(x[len("# record "):]) for x in out.err.splitlines()]
    assert records == entries


def test_one_configuration_alone(capsys):
    bench.report(dict(metric=bench.METRIC), [record("one")])
    out = capsys.readouterr()
    assert json.loads(out.out) == dict(metric=bench.METRIC) and json.loads(out.err[len("# record "):])["workload"] == "one"
