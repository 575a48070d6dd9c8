"""Edges of the paged operators that need no device: status words, descriptors of cut items, arguments, the pool's checks."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_11133_b200", "csrc")


def sources():
    return {os.path.basename(p): open(p).read() for p in glob.glob(os.path.join(CSRC, "*.cu*"))}


def test_no_kernel_reports_an_expired_wait_as_bad_input():
    """The words of the caller's input (a token, an index) are answered as an argument error and taken off the record: a wait that expired
    must not look like one."""
    text = "\n".join(sources().values())
    of_input = {int(v) for v in re.findall(r"constexpr int32_t kStatusBad\w+ = (\d+);", text)}
    waits = [int(v) for v in re.findall(r"abort_flag && \w+\.status\) atomicExch\(\w+\.status, (\d+)\);", text)]
    assert len(of_input) == 2 and len(waits) >= 8
    assert not of_input & set(waits)
