"""Rules of the kernels' sources that no run can show to be kept, checked by reading them."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2509_05512_gb300", "csrc")


def source(name):
    """A source's text without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("name", ["qpoint_f8.cu", "qpoint_f8_tc.cuh", "f8.cuh", "residual.cu",
                                  "philox.cuh", "vec_io.cuh"])
def test_no_load_through_the_read_only_path(name):
    # These grids start while the one before them may still write their inputs, and wait for it
    # inside the kernel.  __ldg and ld.global.nc promise memory that nothing writes while the kernel
    # runs, and such a load may be moved in front of the wait.
    assert not re.search(r"__ldg\b|ld\.global\.nc|const\s+\w+\s*\*\s*__restrict__", source(name))
