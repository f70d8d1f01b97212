"""Barriers that hand a place in LDS from its readers to the loads that refill it, read from the kernels' sources.

Loads that write LDS directly do not go through the compiler's bookkeeping, so the wait in front of such a barrier has to be written out in full: vmcnt for
the loads that the next step reads, and lgkmcnt(0) for the wavefront's own reads of the place that is refilled next.  Without the latter it rests on
where the compiler happens to put its own waits whether a read is still open when another wavefront's load overwrites the place."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2207_09682_amd", "csrc")


def _barriers():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        with open(path) as f:
            for number, line in enumerate(f, 1):
                if "s_barrier" in line and "asm" in line:
                    yield os.path.basename(path), number, line


@pytest.mark.parametrize("header", ["product_device.h", "middle_device.h", "sweep_device.h"])
def test_barriers_wait_for_loads_and_for_the_wavefronts_own_reads(header):
    lines = [(number, line) for name, number, line in _barriers() if name == header]
    assert lines
    for number, line in lines:
        wait = re.search(r's_waitcnt ([^"\\]*)', line)
        assert wait and "lgkmcnt(0)" in wait.group(1), f"{header}:{number}: a barrier that does not wait for LDS reads"
        assert '"memory"' in line, f"{header}:{number}: the compiler may move accesses across it"
