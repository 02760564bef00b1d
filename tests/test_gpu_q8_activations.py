"""silu and gelu behind every tile kernel of the forward products in 8 bits, against 64 bits: biases of their own for both of a pair's products,
what is kept for the backward pass, the residual, and the same call without what is kept."""
import pytest
import torch

from tests import q8_util as ref
from tests.block_util import within
from tests.q8_activation_sizes import SIZES

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


def normal(gen, *shape, std=1.0, dtype=BF16):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%s-%dx%dx%d" % (SIZES[s].replace(" ", "-"), *s[1:]))
def test_forward(tfla, size, kind):
    pair, M, K, N = size
    print(SIZES[size], size, kind, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    act = {"silu": tfla.ACT_SILU, "gelu": tfla.ACT_GELU}[kind]
    # (pre-activations of a few units, to both sides)
    x, w, w2 = ref.to_codes(normal(gen, M, K)), *(ref.to_codes(normal(gen, N, K, std=2 * K ** -0.5), 128) for _ in range(2))
    bias, bias2 = normal(gen, N, std=2.0, dtype=F32), normal(gen, N, dtype=F32) + 0.5
    if pair:
        o = tfla.gated_q8_fwd(*x, *w, *w2, bias, bias2, act=act, keep_pre=True)
        (a, ea), (u, eu), (h, eh) = ref.gated(ref.stands(*x), ref.stands(*w), ref.stands(*w2), bias, bias2, kind)
        within("a", o["a"], a, ea)
        within("u", o["u"], u, eu)
        within("h", o["h"], h, eh)
        ref.coded("hq", o["hq"], o["h_scale"], h, eh)
        lean = tfla.gated_q8_fwd(*x, *w, *w2, bias, bias2, act=act)
        assert same(lean["hq"], o["hq"]) and same(lean["h_scale"], o["h_scale"])
        return
    residual = normal(gen, M, N)
    o = tfla.linear_q8_fwd(*x, *w, bias, residual, act=act, keep_pre=True)
    (z, ez), (y, ey) = ref.linear(ref.stands(*x), ref.stands(*w), bias, residual, kind)
    within("z", o["z"], z, ez)
    within("y", o["y"], y, ey)
    assert same(tfla.linear_q8_fwd(*x, *w, bias, residual, act=act)["y"], o["y"])
