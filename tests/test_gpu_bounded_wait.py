"""The matrix products' bounded wait on the device, and how its running out is told: tests/cuda/bounded_wait.cu, wait_status.cu."""
import os
import subprocess

import pytest

from paper_2006_07405_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(tmp_path, name, *others):
    exe = tmp_path / name
    subprocess.check_call([build.nvcc(), *build.COMPILE_FLAGS, "-I", build.CSRC, "-o", str(exe),
                           os.path.join(ROOT, "tests", "cuda", name + ".cu"), *others])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout + out.stderr


def test_a_wait_that_runs_out_is_given_up_by_whole_warps(tmp_path):
    _run(tmp_path, "bounded_wait")


def test_every_stream_is_told_of_a_wait_that_ran_out(tmp_path):
    _run(tmp_path, "wait_status", os.path.join(build.CSRC, "a2sgd_train.cu"))
