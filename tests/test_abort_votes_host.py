"""How the kernels' roles look at the flag that says that a wait ran out. It may be raised between
the looks of a warp's lanes, so a warp that leaves on it must vote: lanes that stay behind would
wait in the next warp-wide instruction for lanes that are gone, and that wait has no limit. No
call here reaches a kernel."""
import os
import re

import pytest

CSRC = os.path.join("paper_2609_33874_gb300", "csrc")


def _files(root):
    return sorted(f for f in os.listdir(os.path.join(root, CSRC)) if f.endswith((".cu", ".cuh")))


def lone_looks(text):
    """Branches on a lane's own look at the flag. (With `abort &&` before it the look is that of
    the bounded waits, whose outcome the callers share.)"""
    return re.findall(r"(?:if|while) \(\*abort_flag\)", re.sub(r"//[^\n]*", "", text))


def test_no_warp_leaves_on_a_lane_s_own_look(repo_root):
    for f in _files(repo_root):
        with open(os.path.join(repo_root, CSRC, f)) as src:
            assert lone_looks(src.read()) == [], f


@pytest.mark.parametrize("text,n", [
    ("if (*abort_flag) {", 1), ("while (*abort_flag) {}", 1),
    ("if (__any_sync(0xffffffffu, *abort_flag)) {", 0), ("// if (*abort_flag)", 0),
    ("*abort_flag = 1;", 0)])
def test_what_counts_as_a_lone_look(text, n):
    assert len(lone_looks(text)) == n
