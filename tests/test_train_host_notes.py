"""What the training operators' host code keeps between calls, compiled against a runtime of two devices and run without a GPU."""
import os
import subprocess

import pytest

from paper_2006_07405_b200 import build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cuda")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = tmp_path_factory.mktemp("host_notes") / "host_notes"
    lib = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "lib64")   # the program's own functions come before it
    subprocess.check_call([build.nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "shared", "-I", build.CSRC,
                           "-Xlinker", "-rpath=" + lib, "-o", str(exe), os.path.join(HERE, "host_notes.cu"), os.path.join(HERE, "fake_runtime.cpp"),
                           os.path.join(build.CSRC, "a2sgd_train.cu")])
    return exe


def _run(program, part):
    out = subprocess.run([str(program), part], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_every_stream_is_told_of_a_wait_that_ran_out(program):
    """One that another stream's caller asks about, or that runs out between two questions, is lost to nobody."""
    _run(program, "count")


def test_what_fits_on_an_sm_is_noted_for_each_device(program):
    _run(program, "occupancy")
