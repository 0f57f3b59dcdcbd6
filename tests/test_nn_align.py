"""The copy of unaligned operands: which thread takes what, on the host (where a division
by zero ends the program)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_threads_of_a_copy(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "align_check")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-x", "hip", "-O0", "-std=c++17",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2010_13972_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "align_check.cpp"), "-o", exe], check=True,
                   capture_output=True, text=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0, (done.returncode, done.stdout)
