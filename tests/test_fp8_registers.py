"""The sum of two FP8 products on CTA pairs that adds up its accumulators in registers (fp32
outputs of more than 1024 terms) has 128 sums a thread; it has to keep them there.  (No GPU
needed: the compiler says what it spills.)"""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")

from paper_2010_14298_gb300 import build  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "fqt_fp8_core.cuh"
template __global__ void fqt::k_f8_mm<256, 1, true, true, fqt::F8_SUM>(
    const __grid_constant__ fqt::F8Of<fqt::F8_SUM>::Maps, const fqt::F8Of<fqt::F8_SUM>::Args);
"""


@pytest.mark.skipif(not (shutil.which("nvcc") or os.path.exists("/usr/local/cuda/bin/nvcc")),
                    reason="no nvcc")
def test_no_spilled_sums(tmp_path):
    cu = tmp_path / "one.cu"
    cu.write_text(SOURCE)
    r = subprocess.run([build._nvcc(), *build.ARCH, *build.FLAGS, "-Xptxas", "-v", "-c", str(cu), "-o",
                        str(tmp_path / "one.o"), "-I", os.path.join(ROOT, "include"), "-I",
                        os.path.join(ROOT, "paper_2010_14298_gb300", "csrc")],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    said = r.stderr + r.stdout
    spills = [line for line in said.splitlines() if "spill stores" in line]
    assert spills and all("0 bytes spill stores, 0 bytes spill loads" in line for line in spills), said
