"""What can be checked of the cache operators' kernels by their source alone."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_19659_gb300", "csrc")


def test_no_load_by_the_read_only_path():
    """The kernels are launched while the one ahead of them still runs, and that may be an append: loads of what it
    writes (codes, scales, queries) must not go by the path for data that stays as it is while a kernel lives."""
    files = glob.glob(os.path.join(CSRC, "fs_kv*.cu*"))
    assert len(files) == 4
    for f in files:
        with open(f) as s:
            assert not re.search(r"__ldg|ld\.global\.nc|ld\.global\.v4\.nc|__restrict__", s.read()), f
