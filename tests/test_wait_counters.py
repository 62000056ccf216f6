"""Waits that ran out are told of by the operator whose they were: tests/cuda/host_counters.cu (no GPU), wait_status_two.cu."""
import os
import subprocess

import pytest

from paper_2006_07405_b200 import build

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "cuda")
TRAIN = os.path.join(build.CSRC, "a2sgd_train.cu")


def _ok(exe):
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_two_counters_on_one_stream(tmp_path):
    exe = tmp_path / "host_counters"
    lib = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "lib64")   # the program's own functions come before it
    subprocess.check_call([build.nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "shared", "-I", build.CSRC,
                           "-Xlinker", "-rpath=" + lib, "-o", str(exe), os.path.join(HERE, "host_counters.cu"), os.path.join(HERE, "fake_runtime.cpp"), TRAIN])
    _ok(exe)


@pytest.mark.gpu
def test_attention_and_feed_forward_are_told_apart(tmp_path):
    source, part, exe = os.path.join(HERE, "wait_status_two.cu"), tmp_path / "part.o", tmp_path / "wait_status_two"
    first = subprocess.Popen([build.nvcc(), *build.COMPILE_FLAGS, "-DFEED_FORWARD", "-I", build.CSRC, "-c", "-o", str(part), source])
    rest = tmp_path / "rest.o"
    second = subprocess.Popen([build.nvcc(), *build.COMPILE_FLAGS, "-I", build.CSRC, "-c", "-o", str(rest), source])
    assert first.wait() == 0 and second.wait() == 0
    subprocess.check_call([build.nvcc(), *build.COMPILE_FLAGS, "-I", build.CSRC, "-o", str(exe), str(part), str(rest), TRAIN])
    _ok(exe)
