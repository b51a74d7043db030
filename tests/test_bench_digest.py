"""A measured figure on record belongs to the sources of the kernels that it was measured with, and to no other file."""
import json
import os
import shutil
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def test_the_digest_is_of_the_codecs_sources_alone(tmp_path, monkeypatch):
    import bench

    shutil.copytree(bench.CSRC_DIR, tmp_path / "csrc")
    before = bench.csrc_digest()
    monkeypatch.setattr(bench, "CSRC_DIR", str(tmp_path / "csrc"))
    assert bench.csrc_digest() == before
    for other in ("ciera_route.cu", "ciera_fp8.cu", "ciera_numeric.cuh", "something_new.cu"):
        with open(tmp_path / "csrc" / other, "a") as f:
            f.write("// more\n")
    assert bench.csrc_digest() == before
    for name in ("ciera_encode.cu", "ciera_encode_pieces.inc", "ciera_internal.cuh", "ciera_host_step.hpp"):
        was = bench.csrc_digest()
        with open(tmp_path / "csrc" / name, "a") as f:
            f.write("// more\n")
        assert bench.csrc_digest() != was, name


def test_a_figure_is_reported_while_its_sources_stand(tmp_path, monkeypatch):
    import bench

    record = {"some_case": {"dram_bytes_per_value": 4.0, "captured": "here", "csrc_sha256": bench.csrc_digest()}}
    path = tmp_path / "traffic.json"
    path.write_text(json.dumps(record))
    monkeypatch.setattr(bench, "TRAFFIC_FILE", str(path))
    assert bench.measured_traffic("some_case", 100)[0] == 400.0
    record["some_case"]["csrc_sha256"] = "0"
    path.write_text(json.dumps(record))
    assert bench.measured_traffic("some_case", 100)[0] is None
