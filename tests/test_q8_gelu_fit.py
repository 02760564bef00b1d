"""gelu in the backward pass in 8 bits: Phi(-z) = exp(-z^2 / 2) h(z), h by a fit whose constants stand in csrc/q8_quant.hip.  They are taken from
there and compared with 64 bits: as they are, in exact arithmetic, and step by step in fp32 as the kernel goes, with the hardware's reciprocal
right to a unit of its last place."""
import math
import os
import re

import pytest
import torch

from tests.test_block_plan import CSRC

F64 = torch.float64


@pytest.fixture(scope="module")
def constants():
    text = open(os.path.join(CSRC, "q8_quant.hip")).read()
    c = re.search(r"fmaf\((\S+)f, fabsf\(z\), 1\.0f\)", text).group(1)
    p = re.search(r"float P\[9\] = \{(.*?)\};", text).group(1)
    return [fp32(torch.tensor(float(v.strip().rstrip("f")), dtype=F64)) for v in [c] + p.split(",")]


def fp32(v):
    return v.to(torch.float32).to(F64)


def worst(h, z):
    """largest relative error of h, as a power of two"""
    return math.log2(float((h / (0.5 * torch.special.erfcx(z / math.sqrt(2.0))) - 1).abs().max()))


Z = torch.linspace(0, 14.5, 500_001, dtype=F64).to(torch.float32).to(F64)


def test_the_fit(constants):
    c, *p = constants
    t = 1 / (1 + c * Z)
    h = torch.zeros_like(t)
    for k in p[::-1]:
        h = h * t + k
    assert worst(h * t, Z) < -24.2


@pytest.mark.parametrize("off,bits", [(0, -21.3), (1, -20.3), (-1, -20.3)])
def test_the_fit_in_single_precision(constants, off, bits):
    c, *p = constants
    t = fp32(1 / fp32(1 + c * Z))
    t = t + off * torch.exp2(torch.floor(torch.log2(t)) - 23)
    h = p[-1].expand_as(t)
    for k in p[-2::-1]:
        h = fp32(t * h + k)
    assert worst(fp32(t * h), Z) < bits
