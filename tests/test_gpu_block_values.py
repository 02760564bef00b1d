"""Values of the residual block's activations where they are small: relative to what the formula gives, not to the largest value."""
import pytest
import torch

from tests import block_util as bu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


def arguments(dtype):
    """negative values down to where exp(-z^2 / 2), or exp(z), is 1e-33: with z and the derivative's terms no result leaves fp32"""
    z = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(BF16).to(dtype)
    return z[(z < -2.0 ** -20)]


def relative(name, got, terms, err):
    """got against the sum of `terms` (64 bits), each good to `err` of its own size, and half a step"""
    ref = sum(terms)
    lim = err * sum(t.abs() for t in terms)
    lim = lim + bu.HALF[got.dtype] * (ref.abs() + lim)
    bad = ((got.to(bu.F64) - ref).abs() > lim) | ~torch.isfinite(got)
    worst = ((got.to(bu.F64) - ref).abs() / lim).nan_to_num(float("inf")).max()
    assert not bool(bad.any()), "%s: %d of %d off, worst %.3g times the bound" % (name, int(bad.sum()), bad.numel(), float(worst))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_keep_their_digits(tfla, act, dtype):
    """Errors, relative.  The exponential: a rounding of its argument's two products, 2 x 2^-24 of it, so z^2 2^-24 (gelu) and 2 |z| 2^-24
    (silu).  erfc of a rounded argument x (two roundings): 2 x^2 + 1 = z^2 + 1 times 2^-23.  Functions themselves, products and divisions:
    2^-20 (sixteen roundings).  Phi of bf16 tensors: 2^-13 by its statement."""
    z = arguments(dtype)
    z = z[z > (-12.0 if act == "gelu" else -75.0)].contiguous()
    code = tfla.ACT_GELU if act == "gelu" else tfla.ACT_SILU
    x, one = z[:, None].contiguous(), torch.ones((1, 1), dtype=dtype, device="cuda")
    f = tfla.linear_fwd(x, one, act=code, keep_pre=True)
    assert torch.equal(f["z"], x)
    g = tfla.linear_bwd(x, one, torch.ones_like(x), f["z"], act=code, want_dw=False)["dx"][:, 0]
    d = z.to(bu.F64)
    if act == "gelu":
        phi = torch.exp(-0.5 * d * d) / (2 * torch.pi) ** 0.5
        cdf = 0.5 * torch.erfc(-d / 2 ** 0.5)
        err = (d * d + 1) * 2.0 ** -23 + 2.0 ** -20 + (2.0 ** -13 if dtype == BF16 else 0)
        relative("gelu", f["y"][:, 0], [d * cdf], err)
        relative("slope", g, [cdf, d * phi], err)
    else:
        s = torch.sigmoid(d)
        err = 2 * d.abs() * 2.0 ** -24 + 2.0 ** -20
        relative("silu", f["y"][:, 0], [d * s], err)
        relative("slope", g, [s, d * s * (1 - s)], err)
