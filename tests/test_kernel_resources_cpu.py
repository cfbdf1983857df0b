"""Registers that the compiler gives a kernel whose speed stands on the blocks an SM runs at once."""
import os
import re
import subprocess

import pytest

from paper_2509_05512_gb300 import build


def registers(source, tmp_path):
    """{mangled name: registers a thread} of a source's kernels, compiled as the library is."""
    try:
        nvcc = build._nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    r = subprocess.run([nvcc, "-std=c++17", "-O3", *build.ARCH, "-I", build.INCLUDE, "-I", build.CSRC,
                        "--expt-relaxed-constexpr", "-Xptxas", "-v", "-cubin",
                        os.path.join(build.CSRC, source), "-o", str(tmp_path / "out.cubin")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return {m[1]: int(m[2]) for m in
            re.finditer(r"Compiling entry function '(\w+)'.*?Used (\d+) registers", r.stderr, re.S)}


def test_three_blocks_of_the_residual_join_an_sm(tmp_path):
    # The join of aligned bf16 rows, a statistic within a warp: 256 threads a block, and an SM's
    # 65,536 registers go out eight at a time, so three blocks have 80 a thread at most.  (Two blocks
    # an SM: 12% slower, the norm alone 27%.)
    used = registers("residual.cu", tmp_path)
    join = [n for k, n in used.items()
            if "join_fwd_kernelI13__nv_bfloat16Li8ELi1ELb0ELb0EE" in k]
    assert len(join) == 1 and join[0] <= 80
