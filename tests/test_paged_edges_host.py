"""Edges of the paged operators that need no device: status words, descriptors of cut items, arguments, the pool's checks."""
import glob
import os
import re

import pytest

from paper_2602_11133_b200 import build as jot_build

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


@pytest.fixture(scope="module")
def jot():
    jot_build.build()
    from paper_2602_11133_b200 import jot as binding
    binding._lib()
    return binding


def test_scales_whose_exponents_overflow_are_refused(jot):
    """Scores are scaled by scale * log2(e): a finite scale can make it infinite, and zero times it is no number."""
    lib = jot._lib()
    at = 4096                                  # an aligned address that nothing dereferences: the check comes first
    pages = jot._pack_pages(at, at, 0, 0, 4 * 16 * 64, 4 * 16 * 64, 1, 8, 4, 16, 64, 0)

    def call(scale):                           # without a workspace, which is looked at behind the scale
        return lib.jot_paged_attention(at, 256, 256, 64, at, 256, 256, 64, None, 1, 1, 4, pages, 0, at, 4, 4, at, scale, None, 0, None, None)

    assert [call(s) for s in (3e38, -3e38, 2.5e38)] == [-1] * 3
    assert [call(s) for s in (0.0, -0.0, 1e-45, 0.125, -0.125, 2.3e38)] == [-3] * 6
