"""The division by a page's groups that the library's kernels make, compiled for the host from the
library's own header (CPU only)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc is needed to build the helper")
def test_page_of_a_group_is_the_librarys_quotient(tmp_path):
    from paper_2606_03928_amd.build import hipcc
    exe = str(tmp_path / "page_div")
    res = subprocess.run([hipcc(), "-x", "hip", "--cuda-host-only", "-nogpulib", "-O2", "-std=c++17",
                          "-I", os.path.join(ROOT, "include"),
                          "-I", os.path.join(ROOT, "paper_2606_03928_amd", "csrc"),
                          os.path.join(ROOT, "tests", "helpers", "page_div.hip"), "-o", exe],
                         capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-3000:]
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout
    assert int(re.match(r"(\d+) checked, 0 wrong", out.stdout)[1]) > 1000000
