"""Paged key / value cache: what holds on the host, without a device."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_overlapped_kernels_read_through_the_constant_path_only_what_no_launch_writes():
    """A kernel that starts before the one in front of it ends must not read that one's results as read-only memory."""
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2601_17702_b200", "csrc", "*")):
        text = re.sub(r"//.*", "", open(path).read())
        if "cudaGridDependencySynchronize" not in text and "launch_overlapped" not in text:
            continue
        found += 1
        assert "ld.global.nc" not in text and "__restrict__" not in text, path
        for arg in re.findall(r"__ldg\((.*?)[;,]", text):
            assert "cosv" in arg or "sinv" in arg, f"{os.path.basename(path)}: __ldg({arg}"
    assert found >= 5
