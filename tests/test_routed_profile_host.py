"""The summary of the routed layer's kernels carries a fingerprint of the sources that it was taken from, and bench.py reads it."""
import os
import re

import bench


def test_every_routed_source_is_in_one_fingerprint():
    csrc = os.path.join(bench.ROOT, "paper_2403_17017_amd", "csrc")
    assert all(os.path.exists(os.path.join(csrc, n)) for n in bench.ROUTED_SOURCES)
    # what the routed sources include is theirs, common.hiph or the C ABI's header
    for name in bench.ROUTED_SOURCES:
        text = open(os.path.join(csrc, name)).read()
        for inc in re.findall(r'#include "([^"]+)"', text):
            assert os.path.basename(inc) in bench.ROUTED_SOURCES + ("common.hiph", "seer.h"), (name, inc)
    # and no sparse source includes one of them
    for name in set(os.listdir(csrc)) - set(bench.ROUTED_SOURCES):
        if name.endswith((".hip", ".hiph", ".h")):
            assert not set(re.findall(r'#include "([^"]+)"', open(os.path.join(csrc, name)).read())) & set(bench.ROUTED_SOURCES), name


def test_stale_and_fresh(tmp_path):
    f = tmp_path / "summary.txt"
    f.write_text("# kernels\nsource_sha16: 0123456789abcdef\n")
    assert bench.routed_profile(str(f))["stale"] is True
    f.write_text(f"# kernels\nsource_sha16: {bench.routed_source_sha16()}\n")
    assert bench.routed_profile(str(f))["stale"] is False
    f.write_text("# kernels\n")
    assert bench.routed_profile(str(f))["stale"] is True                 # one without a fingerprint is, too
    assert bench.routed_profile(str(tmp_path / "none"))["stale"] is None


def test_the_committed_summary_has_one():
    path = os.path.join(bench.ROOT, "profiles", "kernel_trace_routed.txt")
    assert re.fullmatch("[0-9a-f]{16}", bench._read_summary(path)["source_sha16"])
