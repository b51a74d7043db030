"""The figures on record were measured with the codec's sources as they are: whatever else of the folder changes stays out of the headers that
the codec includes, or the figures are taken again."""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def test_every_figure_on_record_is_of_the_sources_that_are_here():
    import bench

    with open(bench.TRAFFIC_FILE) as f:
        record = {k: v for k, v in json.load(f).items() if not k.startswith("_")}
    assert record and {v["csrc_sha256"] for v in record.values()} == {bench.csrc_digest()}
    assert bench.measured_traffic("encode_exact_bf16_B512_clustered_f0.22", 1000)[0] is not None
