"""The runtime starts fewer than 2^32 threads along an axis.  At the largest sizes that the calls in 8 bits accept, no launch asks for more, nor
does the launch of both backward products in bf16: the rules (csrc/q8_plan.h, gemm_plan.h, the headers that the library is built with) compiled
for the host."""
import ctypes
import itertools
import os
import subprocess

import pytest

from tests.test_block_plan import CSRC, HERE

LIMIT = 1 << 32


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("launch") / "q8_launch.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, os.path.join(HERE, "q8_launch_probe.cpp"), "-o", so])
    return ctypes.CDLL(so)


@pytest.mark.parametrize("more", [0, 1, 256, (1 << 14) + 256, 1 << 22])
@pytest.mark.parametrize("M,N", [(1, 1), (128, 129), (1 << 24, 3968), (1 << 24, 3969), (1 << 24, 4096), (1 << 18, 1 << 18), (1 << 16, 1 << 20), (1 << 21, 1 << 15),
                                 ((1 << 24) - 1, 4095), ((1 << 21) - 5, (1 << 15) - 200)])
def test_tiles(probe, M, N, more):
    """all workgroups, in order, in launches that the runtime accepts; each begins at a multiple of eight, as XCDs are counted"""
    ask = probe.tile_launches
    ask.argtypes = [ctypes.c_long, ctypes.c_long, ctypes.c_uint, ctypes.POINTER(ctypes.c_long), ctypes.POINTER(ctypes.c_long)]
    first, threads = (ctypes.c_long * 64)(), (ctypes.c_long * 64)()
    n = ask(M, N, more, first, threads)
    at = 0
    for i in range(n):
        assert first[i] == at and at % 8 == 0 and 0 < threads[i] < LIMIT
        at += threads[i] // 1024
    assert at == -(-M // 128) * -(-N // 128) + more
    if at < 1 << 21:
        assert n == 1


def sizes(most):
    """powers of two up to the limit and what lies next to them"""
    return sorted({n for p in range(0, most + 1, 2) for n in (1 << p, (1 << p) + 1, (3 << p) // 2) if n <= 1 << most} | {1 << most, (1 << most) - 1})


@pytest.mark.parametrize("backward,pair", itertools.product((0, 1), (0, 1)))
def test_products(probe, backward, pair):
    ask = probe.product_threads
    ask.argtypes, ask.restype = [ctypes.c_int] * 2 + [ctypes.c_long] + [ctypes.c_int] * 2, ctypes.c_long
    worst = (0,)
    for M, K, N in itertools.product(sizes(21 if backward else 24), sizes(20), sizes(20)):
        if max(M * K, M * N, N * K) <= 1 << 36:
            worst = max(worst, (ask(backward, pair, M, K, N), M, K, N))
    # the weights' size limit itself, in every proportion
    for i in range(1 << 16, (1 << 20) + 1, 997):
        for K, N in ((i, (1 << 36) // i), ((1 << 36) // i, i)):
            if max(K, N) <= 1 << 20:
                worst = max(worst, *((ask(backward, pair, M, K, N), M, K, N) for M in (1, 5, 40, 64, 128)))
    assert worst[0] < LIMIT, worst


@pytest.mark.parametrize("pair", (0, 1))
def test_both_products_in_bf16(probe, pair):
    ask = probe.both_items
    ask.argtypes, ask.restype = [ctypes.c_int, ctypes.c_long, ctypes.c_int, ctypes.c_int], ctypes.c_long
    most = max(ask(pair, M, K, N) for M, K, N in itertools.product(sizes(24), sizes(20), sizes(20)) if max(M * K, M * N, N * K) <= 1 << 36)
    assert 0 < most < LIMIT // 256
