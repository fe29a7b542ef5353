"""The paged cache's kernels are set up while the grid before them is still at work and may write what they are to read.  The read-only path is for memory that
nobody writes while a grid lives, so none of their loads goes through it: read from the sources, since a stale value would be a matter of luck."""
import glob
import os
import re

import pytest

from tests.test_bounded_waits_cpu import CSRC

SOURCES = sorted(glob.glob(os.path.join(CSRC, "paged*")))
READ_ONLY = re.compile(r"\b__ldg\s*\(|\.nc\b|__restrict__|\btex\w*D\s*<")


def code(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def test_the_kernels_are_found():
    assert {os.path.basename(p) for p in SOURCES} >= {"paged.cu", "paged_store.cuh", "paged_stream.cuh", "paged_tile.cuh", "paged_view.cuh"}
    assert "cudaLaunchAttributeProgrammaticStreamSerialization" in code(os.path.join(CSRC, "paged.cu"))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_load_by_the_read_only_path(path):
    assert READ_ONLY.findall(code(path)) == []
