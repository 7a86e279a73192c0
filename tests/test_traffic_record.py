"""The committed HBM traffic record is of the kernel sources as they are: the benchmark
reports its figures only then."""

import json

import bench


def test_the_record_is_current():
    with open(bench.TRAFFIC_FILE) as f:
        rec = json.load(f)
    assert rec["kernel_source_sha256"] == bench.kernel_source_hash(), (
        "the kernel sources changed: take the counters again and write the record with "
        "`bench.py --write-traffic-record`")
    assert bench.recorded_traffic() == rec["bwd_bytes_per_launch"] > 0
    assert bench.recorded_decode_traffic() == rec["decode_bytes_per_step"] > 0
