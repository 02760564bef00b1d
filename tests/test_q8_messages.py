"""What the binding says of tensors that the calls in 8 bits refuse names the types that they take."""
import pytest
import torch

import paper_2503_14376_amd as tfla
from tests.test_block_arguments import lib  # noqa: F401


def test_gradients_in_single_precision(lib):  # noqa: F811
    x, q, s = torch.zeros(4, 8), torch.zeros(8, 8).to(torch.float8_e4m3fn), torch.ones(1, 1).to(torch.float8_e8m0fnu)
    for call in (lambda: tfla.linear_q8_bwd(x, q, s, x), lambda: tfla.gated_q8_bwd(x, q, s, q, s, x, x, x)):
        with pytest.raises(ValueError, match=r"must be bfloat16 \(got torch.float32\)"):
            call()
    for call in (lambda: tfla.q8_quant(x.half()), lambda: tfla.norm_q8_fwd(x.half())):
        with pytest.raises(ValueError, match=r"must be bfloat16 or float32 \(got torch.float16\)"):
            call()
