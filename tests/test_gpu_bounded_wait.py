"""The matrix products' bounded wait on the device: tests/cuda/bounded_wait.cu."""
import os
import subprocess

import pytest

from paper_2006_07405_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_wait_that_runs_out_is_given_up_by_whole_warps(tmp_path):
    exe = tmp_path / "bounded_wait"
    subprocess.check_call([build.nvcc(), *build.COMPILE_FLAGS, "-I", build.CSRC, "-o", str(exe),
                           os.path.join(ROOT, "tests", "cuda", "bounded_wait.cu")])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout + out.stderr
