"""What can be checked of the products' kernels by their source alone."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_19659_gb300", "csrc")


def sources():
    files = glob.glob(os.path.join(CSRC, "fs_mm*.cu*"))
    assert len(files) == 4
    return {os.path.basename(f): open(f).read() for f in files}


def test_no_load_by_the_read_only_path():
    """The kernels are launched while the one ahead of them still runs, and that may write what they read."""
    for name, text in sources().items():
        assert not re.search(r"__ldg|ld\.global\.nc|__restrict__", text), name


def test_tensor_memory_is_asked_for_after_the_kernels_ahead():
    """A block that held some while it waits for a kernel ahead, whose blocks may still ask for all of it, would wait for
    ever. (k_mm_wide's blocks leave no room for others beside them, so theirs may come first.)"""
    text = sources()["fs_mm_few.cu"]
    assert text.count("tcgen05.alloc") == 1 and text.index("pdl_wait();") < text.index("tcgen05.alloc")
    assert text.index("tcgen05.dealloc") < text.index("cluster_all();  // (the last")
