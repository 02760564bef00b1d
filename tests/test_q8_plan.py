"""Every kernel that the rules for products in 8 bits can choose is among those that the GPU tests run: the rules (csrc/q8_plan.h, the header
that the library is built with) compiled for the host and asked for a grid of sizes and for the tests' own."""
import ctypes
import itertools
import os
import subprocess

import pytest

from tests.q8_sizes import SIZES
from tests.test_block_plan import CSRC, GRID, HERE


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plan") / "q8_plan.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, os.path.join(HERE, "q8_plan_probe.cpp"), "-o", lib])
    ask = ctypes.CDLL(lib).product_kernels
    ask.argtypes = [ctypes.c_int] * 2 + [ctypes.c_long] + [ctypes.c_int] * 2 + [ctypes.c_char_p]
    ask.restype = None
    buf = ctypes.create_string_buffer(1024)

    def names(*case):
        ask(*case, buf)
        return buf.value.decode().split("\n")[:-1]
    return names


def test_the_gpu_tests_reach_every_kernel(kernels):
    run = {k for case in SIZES for k in kernels(*case)}
    missing = {}
    for case in itertools.product((0, 1), (0, 1), GRID, GRID, GRID):
        for k in kernels(*case):
            if k not in run:
                missing.setdefault(k, case)
    assert not missing, "no size in tests/q8_sizes.py reaches: %s" % missing
    assert len(run) >= 150


def test_kernels_differ_by_size_and_direction(kernels):
    """what the names stand for, at sizes whose kernel follows from the rules' text"""
    assert kernels(0, 0, 1, 4096, 4096) == ["rows blocks 1 slices 4 waves 4 ahead 2"]
    assert kernels(0, 1, 4, 4096, 10944) == ["rows pair blocks 1 slices 4 waves 4 ahead 2 hold"]
    assert kernels(0, 1, 8192, 4096, 10944) == ["fwd pair 256x256 many"]
    assert kernels(1, 0, 8192, 4096, 4096) == ["dx 256x256 many", "dw 256x256"]
    assert kernels(1, 1, 1000, 1000, 1365) == ["both pair many"]
