"""The HBM traffic that the benchmark reports comes from a committed profile and holds only for the
decode kernel it was taken on."""
import os
import re

import bench


def test_every_decode_source_counts():
    """The hash that ties the profile to the kernel covers every file of it, headers of headers too."""
    csrc = os.path.dirname(bench.DECODE_SOURCES[0])
    seen, todo = set(), ["mkv_decode.hip"]
    while todo:
        f = todo.pop()
        if f in seen or not os.path.exists(os.path.join(csrc, f)):
            continue
        seen.add(f)
        with open(os.path.join(csrc, f)) as fh:
            todo += re.findall(r'^#include "([\w.]+)"', fh.read(), re.M)
    assert {os.path.basename(f) for f in bench.DECODE_SOURCES} == seen
