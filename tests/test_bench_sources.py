"""The sources that a flow workload's profile is taken on (CPU): all that its
kernels' object is compiled from, so that none can change under a kept profile."""
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2609_35115_amd", "csrc")


def included(name, seen):
    if name in seen or not os.path.exists(os.path.join(CSRC, name)):
        return seen
    seen.add(name)
    for x in re.findall(r'^\s*#include "([^"]+)"', open(os.path.join(CSRC, name)).read(), re.M):
        included(x, seen)
    return seen


def test_flow_sources_are_all_that_is_compiled():
    assert set(bench.FLOW_SOURCES) == included("flow_kernels.hip", set())


def test_a_changed_header_makes_a_profile_stale(tmp_path, monkeypatch):
    for f in bench.FLOW_SOURCES:
        os.makedirs(tmp_path / "paper_2609_35115_amd" / "csrc", exist_ok=True)
        (tmp_path / "paper_2609_35115_amd" / "csrc" / f).write_bytes(open(os.path.join(CSRC, f), "rb").read())
    before = bench.kernel_source_hash(bench.FLOW_SOURCES)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_source_hash(bench.FLOW_SOURCES) == before
    for f in bench.FLOW_SOURCES:
        p = tmp_path / "paper_2609_35115_amd" / "csrc" / f
        old = p.read_bytes()
        p.write_bytes(old + b"\n")
        assert bench.kernel_source_hash(bench.FLOW_SOURCES) != before, f
        p.write_bytes(old)
