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


def test_the_8_bit_product_drains_after_its_roles():
    # A role that has nothing left to do may leave before another one gives up, with its copies or
    # products still under way.  So they are waited for behind the barrier that ends the roles, where
    # the abort flag is final, and in front of the release of TMEM.
    text = source("qpoint_f8_tc.cuh")
    roles_end = text.index("__syncthreads();", text.index("setmaxnreg.inc"))
    flag = text.index("if (*abort_flag)", roles_end)
    release = text.index("tmem_dealloc", flag)
    drains = [m.start() for m in re.finditer(r"drain_fills\(|umma_commit\(drain_bar", text)]
    assert len(drains) == 3 and all(flag < d < release for d in drains)
    # nobody releases anything before the drains have ended
    assert "__syncthreads();" in text[max(drains):release]
