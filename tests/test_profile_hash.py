"""The hash that says which sources a profile was taken on."""
import os

import bench
from paper_2603_04800_amd import build


def test_hash_covers_what_the_library_is_built_from():
    covered = {os.path.basename(f) for f in bench.KERNEL_SOURCES}
    assert set(build.SOURCES) <= covered
    for src in build.SOURCES + tuple(f for f in os.listdir(build.CSRC) if f.endswith(".h")):
        with open(os.path.join(build.CSRC, src)) as f:
            used = [line.split('"')[1] for line in f if line.startswith('#include "')]
        assert {h for h in used if h != "masq.h"} <= covered, (src, used)
    assert all(os.path.exists(os.path.join(bench.ROOT, f)) for f in bench.KERNEL_SOURCES)
    assert len(bench.kernel_source_hash()) == 16
