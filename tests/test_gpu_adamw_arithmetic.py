"""The roots, quotients and codes that AdamW's step writes out for pairs of elements, compared on the device with the single
correctly rounded operations (tests/cuda/adamw_arithmetic.cu): no difference is allowed."""
import os
import subprocess

import pytest

from paper_2006_07405_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pairs_against_single_operations(tmp_path):
    exe = tmp_path / "adamw_arithmetic"
    subprocess.check_call([build.nvcc(), *build.COMPILE_FLAGS, "-I", build.CSRC, "-o", str(exe),
                           os.path.join(ROOT, "tests", "cuda", "adamw_arithmetic.cu")])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    assert [line.split(": ")[1] for line in out.stdout.splitlines()] == ["0 differences"] * 4, out.stdout
