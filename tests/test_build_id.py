"""Which sources a measurement belongs to: the whole library's, or the cache's alone."""
import json
import os
import re

import bench
from paper_2112_07221_amd import build
from paper_2112_07221_amd import hetcache as hc


def test_the_caches_sources_do_not_include_the_dense_layers():
    for name in os.listdir(build.CSRC):
        if not name.startswith("dense"):
            text = open(os.path.join(build.CSRC, name)).read()
            assert not re.search(r"#include\s*[<\"][^>\"]*dense", text), name


def test_the_caches_id_is_its_sources_alone(tmp_path, monkeypatch):
    for n in os.listdir(build.CSRC):
        (tmp_path / n).write_bytes(open(os.path.join(build.CSRC, n), "rb").read())
    whole, cache = build.source_id(), build.cache_id()
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    assert (build.source_id(), build.cache_id()) == (whole, cache)
    (tmp_path / "dense_types.hpp").write_text("// other layers\n")
    (tmp_path / "dense_more.hpp").write_text("// and more of them\n")
    assert build.source_id() != whole and build.cache_id() == cache
    (tmp_path / "common.hpp").write_text("// another cache\n")
    assert build.cache_id() != cache


def test_recorded_traffic_is_given_for_the_same_cache(tmp_path, monkeypatch):
    record = tmp_path / "traffic.json"
    monkeypatch.setattr(bench, "TRAFFIC_FILE", str(record))
    monkeypatch.setattr(hc, "build_id", build.source_id)
    entry = {"cache_id": build.cache_id(), "bytes_per_launch": {"apply_kernel": 5}}
    record.write_text(json.dumps({"config2": entry, "config4": {**entry, "cache_id": "other"}}))
    assert bench.measured_traffic("apply_kernel", 2) == 5
    assert bench.measured_traffic("probe_kernel", 2) is None and bench.measured_traffic("apply_kernel", 4) is None
    assert bench.measured_traffic("apply_kernel", 1) is None
    monkeypatch.setattr(hc, "build_id", lambda: "another build")
    assert bench.measured_traffic("apply_kernel", 2) is None
    record.unlink()
    assert bench.measured_traffic("apply_kernel", 2) is None
