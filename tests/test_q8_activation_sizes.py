"""The sizes at which activations are compared with 64 bits reach the kernels that they stand for."""
import pytest

from tests.q8_activation_sizes import SIZES
from tests.test_q8_plan import kernels  # noqa: F401


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_kernel(kernels, size):  # noqa: F811
    assert kernels(0, *size) == [SIZES[size]]
