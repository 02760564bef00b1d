"""Tensors of more than 2^31 elements in every place that the residual block's operators read or write one.  All values are small whole
numbers, so that every sum is exact in fp32 and every result in bf16 (to 256 in magnitude): results are compared for equality.  Gradients of
weights and biases come from a few rows, on both sides of 2^30 and 2^31 elements and at both ends, that no other row can make up for."""
import pytest
import torch

from tests.test_gpu_block import BF16, F32

pytestmark = pytest.mark.gpu
M, WIDE = 540_000, 4008


@pytest.fixture(scope="module")
def tfla():
    import paper_2503_14376_amd as pkg
    pkg.load_library()
    return pkg


@pytest.fixture(autouse=True)
def freed():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def whole(seed, rows, cols, dtype, most=2):
    """random whole numbers from -most to most, some rows at a time (no larger tensor of another type on the way)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty((rows, cols), dtype=dtype, device="cuda")
    for lo in range(0, rows, 60_000):
        part = t[lo:lo + 60_000]
        part.copy_(torch.randint(-most, most + 1, part.shape, generator=gen, device="cuda", dtype=torch.int8))
    return t


def far_rows(rows, cols):
    r = [0, 1, rows - 2, rows - 1]
    for at in (1 << 30, 1 << 31):
        r += [at // cols - 1, at // cols, at // cols + 1]
    return torch.tensor(sorted(r), device="cuda")


def few(seed, rows, cols, dtype):
    """zero but in the far rows; the rows differ"""
    t = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    at = far_rows(rows, cols)
    t[at] = whole(seed, len(at), cols, dtype)
    return t, at


def same(got, want, lo=0):
    """a block of rows against fp64"""
    assert torch.equal(got[lo:lo + want.shape[0]].double(), want), lo


def blocks(rows):
    return [(lo, min(rows, lo + 60_000)) for lo in range(0, rows, 60_000)]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_results(tfla, dtype):
    """y and z written, the residual read"""
    print("far forward results", dtype, flush=True)
    x, w = whole(1, M, 32, dtype), whole(2, WIDE, 32, dtype, 1)
    res = whole(3, M, WIDE, dtype)
    f = tfla.linear_fwd(x, w, residual=res, act=tfla.ACT_RELU, keep_pre=True)
    for lo, hi in blocks(M):
        z = x[lo:hi].double() @ w.double().t()
        same(f["z"], z, lo)
        same(f["y"], z.clamp_min(0) + res[lo:hi].double(), lo)
    del f, res
    w2 = whole(4, WIDE, 32, dtype, 1)
    w2[:, 3:] = 0                                            # (the products stay below 256)
    x.clamp_(-1, 1)
    f = tfla.gated_fwd(x, w, w2, act=tfla.ACT_RELU, keep_pre=True)
    for lo, hi in blocks(M):
        a, u = (x[lo:hi].double() @ t.double().t() for t in (w, w2))
        same(f["a"], a, lo)
        same(f["u"], u, lo)
        same(f["h"], a.clamp_min(0) * u, lo)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_input(tfla, dtype):
    print("far forward input", dtype, flush=True)
    x, w = whole(5, M, WIDE, dtype, 1), torch.zeros((40, WIDE), dtype=dtype, device="cuda")
    w[:, ::37] = whole(6, 40, (WIDE + 36) // 37, dtype, 1)
    y = tfla.linear_fwd(x, w)["y"]
    for lo, hi in blocks(M):
        same(y, x[lo:hi].double() @ w.double().t(), lo)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_backward_gradients_of_results(tfla, dtype, act):
    """dy and z read, dz written and read as either operand, the bias sums"""
    print("far backward results", dtype, act, flush=True)
    K = 64
    dy, at = few(7, M, WIDE, dtype)
    x, w = whole(8, M, K, dtype), torch.zeros((WIDE, K), dtype=dtype, device="cuda")
    w[::37] = whole(9, (WIDE + 36) // 37, K, dtype, 1)
    dz = dy[at].double()
    z = None
    if act == "relu":
        z = whole(10, M, WIDE, dtype)
        dz = dz * (z[at] > 0)
    g = tfla.linear_bwd(x, w, dy, z, act=tfla.ACT_RELU if z is not None else tfla.ACT_NONE, want_db=True)
    assert torch.equal(g["dw"].double(), dz.t() @ x[at].double())
    assert torch.equal(g["db"].double(), dz.sum(0))
    assert torch.equal(g["dx"][at].double(), dz @ w.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_of_the_pair(tfla, dtype):
    print("far backward pair", dtype, flush=True)
    K = 64
    dh, at = few(11, M, WIDE, dtype)
    x = whole(12, M, K, dtype, 1)
    wg, wu = (torch.zeros((WIDE, K), dtype=dtype, device="cuda") for _ in range(2))
    wg[::97], wu[1::97] = whole(13, len(range(0, WIDE, 97)), K, dtype, 1), whole(14, len(range(1, WIDE, 97)), K, dtype, 1)
    a, u = whole(15, M, WIDE, dtype), whole(16, M, WIDE, dtype)
    g = tfla.gated_bwd(x, wg, wu, a, u, dh, act=tfla.ACT_RELU, want_db=True)
    d, av, uv = dh[at].double(), a[at].double(), u[at].double()
    da, du = d * uv * (av > 0), d * av.clamp_min(0)
    assert torch.equal(g["dw_gate"].double(), da.t() @ x[at].double()) and torch.equal(g["dw_up"].double(), du.t() @ x[at].double())
    assert torch.equal(g["db_gate"].double(), da.sum(0)) and torch.equal(g["db_up"].double(), du.sum(0))
    assert torch.equal(g["dx"][at].double(), da @ wg.double() + du @ wu.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [0, 1])
def test_backward_gradients_of_inputs(tfla, dtype, shift):
    """dx written; x read in the weights' gradient, in place and as a copy (bf16 off 16 bytes)"""
    print("far backward inputs", dtype, shift, flush=True)
    N = 40
    at = far_rows(M, WIDE)
    x = torch.empty(M * WIDE + 8, dtype=dtype, device="cuda")[shift:shift + M * WIDE].view(M, WIDE)
    x.copy_(whole(17, M, WIDE, dtype))
    w, dy = whole(18, N, WIDE, dtype, 1), torch.zeros((M, N), dtype=dtype, device="cuda")
    dy[at] = whole(19, len(at), N, dtype)
    g = tfla.linear_bwd(x, w, dy)
    assert torch.equal(g["dw"].double(), dy[at].double().t() @ x[at].double())
    assert torch.equal(g["dx"][at].double(), dy[at].double() @ w.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layer", [False, True])
def test_norm_gradients(tfla, dtype, layer):
    """with statistics of 1 (and 0): x^ is x.  The row's means are the only fractions: dx is compared by differences of whole numbers"""
    print("far norm", dtype, layer, flush=True)
    rows, D = 1_050_000, 2056
    dy, at = few(20, rows, D, dtype)
    x = whole(21, rows, D, dtype)
    stat, zero = torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda")
    kind = tfla.NORM_LAYER if layer else tfla.NORM_RMS
    g = tfla.norm_bwd(x, dy, stat, zero, norm_kind=kind, want_dbeta=True)
    d, xv = dy[at].double(), x[at].double()
    assert torch.equal(g["dgamma"].double(), (d * xv).sum(0))
    assert torch.equal(g["dbeta"].double(), d.sum(0))
    want = d - xv * (d * xv).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if layer else 0)
    # (half a step of at most 2 x 2, and some fp32 roundings of terms below 8)
    assert float((g["dx"][at].double() - want).abs().max()) <= 8 * (2.0 ** -8 if dtype == BF16 else 2.0 ** -22)
    g["dx"][at] = 0
    assert not g["dx"].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens", [2, 40])
def test_weights(tfla, dtype, tokens):
    """weights and their gradients, by the kernel for few rows and by tiles"""
    print("far weights", dtype, tokens, flush=True)
    N, K = 1 << 20, 2056
    x = torch.zeros((tokens, K), dtype=dtype, device="cuda")
    x[:, ::37] = whole(22, tokens, (K + 36) // 37, dtype, 1)
    w, at = few(23, N, K, dtype)
    y = tfla.linear_fwd(x, w)["y"]
    assert torch.equal(y[:, at].double(), x.double() @ w[at].double().t())
    y[:, at] = 0
    assert not y.any()
    if tokens == 2:
        h = tfla.gated_fwd(x, w, w, act=tfla.ACT_RELU)["h"]
        assert torch.equal(h[:, at].double(), (x.double() @ w[at].double().t()).clamp_min(0) ** 2)
        del h
    dy = torch.zeros((tokens, N), dtype=dtype, device="cuda")
    dy[:, at] = whole(24, tokens, len(at), dtype, 1)
    g = tfla.linear_bwd(x, w, dy)
    assert torch.equal(g["dx"].double(), dy[:, at].double() @ w[at].double())
    assert torch.equal(g["dw"][at].double(), dy[:, at].double().t() @ x.double())
    g["dw"][at] = 0
    assert not g["dw"].any()
