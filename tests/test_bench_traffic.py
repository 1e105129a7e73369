"""Which sources the benchmark takes for the step's kernels, and that the measured traffic in profiles/ applies to them (CPU)."""
import json
import os
import re

import bench


def _table():
    return json.loads("".join(line for line in open(bench.TRAFFIC_TABLE) if not line.startswith("#")))


def test_the_measured_traffic_is_found():
    for e in _table():
        found, text = bench.load_traffic(e["workload"], e["B"], [o["op"] for o in e["ops"]], [o["pipe"] for o in e["ops"]])
        assert found is not None, (e["workload"], text)
        assert {n: o["hbm_kib"] for n, o in found.items()} == {o["op"]: o["hbm_kib"] for o in e["ops"]}


def test_operators_that_no_step_launches_do_not_count(tmp_path, monkeypatch):
    """Found by what a file includes, itself or through another header."""
    csrc = tmp_path / "paper_2006_11751_amd" / "csrc"
    csrc.mkdir(parents=True)
    (tmp_path / "include").mkdir()
    (tmp_path / "include" / "sf_policy.h").write_text("// policy\n")
    (tmp_path / "include" / "sf_memory.h").write_text("// memory\n")
    for name, text in (("k_step.hip", '#include "sf_shared.h"\n'), ("sf_shared.h", "#pragma once\n"), ("k_direct.hip", '#include "sf_memory.h"\n'),
                       ("sf_near.h", '#include "sf_memory.h"\n'), ("sf_far.h", '#include "sf_near.h"\n'),
                       ("k_far.hip", '#include "sf_shared.h"\n  #  include "sf_far.h"  // (spaces)\n')):
        (csrc / name).write_text(text)
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    before = bench.source_hash()
    for name in ("k_direct.hip", "sf_near.h", "sf_far.h", "k_far.hip"):
        with open(csrc / name, "a") as f:
            f.write("// changed\n")
        assert bench.source_hash() == before, name
    for name in ("k_step.hip", "sf_shared.h"):
        with open(csrc / name, "a") as f:
            f.write("// changed\n")
        after = bench.source_hash()
        assert after != before, name
        before = after


def test_every_operator_of_the_memory_header_is_left_out():
    """A file that has one of its entry points, and no other, is none of the step's."""
    csrc = os.path.join(bench.ROOT, "paper_2006_11751_amd", "csrc")
    names = re.findall(r"^\w+ (sf_\w+)\(", open(os.path.join(bench.ROOT, "include", "sf_memory.h")).read(), re.M)
    assert "sf_deltarule" in names and "sf_gradclip" in names
    out = bench.operator_sources(csrc)
    for name in sorted(os.listdir(csrc)):
        text = open(os.path.join(csrc, name)).read()
        assert name in out or not any('extern "C" int %s(' % n in text for n in names), name
    assert "sf_api.hip" not in out and "sf_internal.h" not in out and "sf_split.h" not in out
