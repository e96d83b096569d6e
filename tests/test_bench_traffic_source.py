"""The DRAM figure that bench.py quotes belongs to one kernel source: all files that the kernel is made of."""
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
CSRC = os.path.join(ROOT, "paper_2105_09377_b200", "csrc")


@pytest.mark.parametrize("name,counts", [
    ("gl_dot.cu", True), ("gl_tc.cuh", True), ("gl_tmap.h", True), ("gl_launch.cuh", True), ("gl_internal.h", True),
    ("gl_mx4.cu", False), ("gl_attend.cu", False), ("gl_memops.cu", False)])
def test_a_change_of_a_file_of_the_kernel_changes_the_key(tmp_path, name, counts):
    import bench
    copy = str(tmp_path / "csrc")
    shutil.copytree(CSRC, copy)
    before = bench.kernel_source_key(os.path.join(copy, "gl_dot.cu"))
    assert before == bench.kernel_source_key(os.path.join(CSRC, "gl_dot.cu"))
    with open(os.path.join(copy, name), "a") as f:
        f.write("\n// changed\n")
    assert (bench.kernel_source_key(os.path.join(copy, "gl_dot.cu")) != before) == counts
