"""The causal mask of the keys kernel over pages, its expression on the host: positions up to the last that a layer may have."""
import os
import shutil
import subprocess

import pytest

from paper_2605_12825_b200.build import NVCC_FLAGS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_12825_b200", "csrc")
NVCC = os.environ.get("NVCC", "nvcc")

PROGRAM = """
#include <cstdio>
#include "paged.cuh"
int main()
{
    int key, pos0, G;
    while (std::scanf("%d %d %d", &key, &pos0, &G) == 3) std::printf("%d\\n", orthrus::rows_before_key(key, pos0, G));
}
"""


@pytest.mark.skipif(shutil.which(NVCC) is None, reason="no CUDA compiler")
def test_far_keys_are_seen_by_all_rows(tmp_path):
    """Row r is at position pos0 + r / G and sees key t if t <= that: in front of the first such row are max(0, t - pos0) G rows."""
    src, exe = tmp_path / "mask.cu", tmp_path / "mask"
    src.write_text(PROGRAM)
    subprocess.run([NVCC, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", str(exe), str(src)], check=True)
    cases = []
    for G in (1, 3, 16, 64, 128):
        for pos0 in (0, 1, 63, 64, 2 ** 31 // G - 1 if G > 1 else 2 ** 30, 2 ** 31 // G + 1 if G > 1 else 2 ** 30, 3 * 2 ** 24, 2 ** 31 - 2 ** 16 - 64):
            for key in {0, 1, pos0 // 2, max(pos0 - 2 ** 24, 0), max(pos0 - 2 ** 24 - 1, 0), max(pos0 - 1, 0), pos0, pos0 + 1, pos0 + 63}:
                cases.append((key, pos0, G))
    out = subprocess.run([str(exe)], input="".join("%d %d %d\n" % c for c in cases), stdout=subprocess.PIPE, check=True, text=True).stdout.split()
    assert [int(x) for x in out] == [max(0, key - pos0) * G for key, pos0, G in cases]
