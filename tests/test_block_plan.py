"""Every kernel that the products' rules can choose is among those that the GPU tests run: the rules (csrc/gemm_plan.h, the header that the
library is built with) compiled for the host and asked for a grid of sizes and for the tests' own."""
import ctypes
import itertools
import os
import subprocess

import pytest

from tests.block_sizes import SIZES

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2503_14376_amd", "csrc")
GRID = (1, 2, 4, 5, 8, 13, 16, 17, 24, 32, 33, 47, 64, 65, 97, 128, 191, 256, 333, 512, 703, 1000, 1365, 2000, 2752, 4096, 5200, 8192, 10944,
        16384, 16700)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, os.path.join(HERE, "gemm_plan_probe.cpp"), "-o", lib])
    ask = ctypes.CDLL(lib).product_kernels
    ask.argtypes = [ctypes.c_int] * 3 + [ctypes.c_long] + [ctypes.c_int] * 2 + [ctypes.c_char_p]
    ask.restype = None
    buf = ctypes.create_string_buffer(1024)

    def names(*case):
        ask(*case, buf)
        return buf.value.decode().split("\n")[:-1]
    return names


def test_the_gpu_tests_reach_every_kernel(kernels):
    run = {k for case in SIZES for k in kernels(*case)}
    missing = {}
    for case in itertools.product((0, 1), (0, 1), (0, 1), GRID, GRID, GRID):
        for k in kernels(*case):
            if k not in run:
                missing.setdefault(k, case)
    assert not missing, "no size in tests/block_sizes.py reaches: %s" % missing
    assert len(run) >= 200


def test_kernels_differ_by_size_type_and_direction(kernels):
    """what the names stand for, at sizes whose kernel follows from the rules' text"""
    assert kernels(0, 1, 0, 1, 4096, 4096) == ["rows bf16 blocks 1 slices 1 waves 8"]
    assert kernels(0, 1, 1, 8192, 4096, 10944) == ["fwd bf16 pair 256x256 many"]
    assert kernels(1, 1, 0, 8192, 4096, 4096) == ["dx bf16 256x256 many", "dw bf16 256x256"]
    assert len(kernels(1, 1, 0, 70, 133, 555)) == 1
