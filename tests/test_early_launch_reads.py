"""Kernels that are launched early run beside the kernel ahead of them in the stream, which may still be writing what they read behind their wait.

The read-only path (__ldg, ld.global.nc, const __restrict__) is for memory that nothing writes while the kernel is there, so none of the sources
may use it.  No run shows the difference reliably: the sources are read."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_12825_b200", "csrc")


def test_no_kernel_reads_by_the_read_only_path():
    files = glob.glob(os.path.join(CSRC, "*.cu*"))
    assert len(files) > 10
    for path in files:
        text = re.sub(r"//[^\n]*", "", open(path).read())
        bad = re.search(r"__ldg\b|\bld(?:\.\w+)*\.nc\b|__restrict__", text)
        assert bad is None, (os.path.basename(path), bad.group(0))
