"""Codes, scales and bf16 tensors of more than 2^31 and 2^32 elements in every place that the calls in 8 bits read or write one.  All values are
small whole numbers (times a power of two codes of their own), so that quantisation and every sum are exact and results have one rounding
to bf16.  Gradients of weights and biases come from a few rows, on both sides of 2^30, 2^31 and 2^32 elements and at both ends, that no
other row can make up for."""
import pytest
import torch

from tests.test_gpu_block import BF16, F32
from tests.test_gpu_block_far import blocks, freed, tfla, whole  # noqa: F401

pytestmark = pytest.mark.gpu
M, WIDE, EVEN = 1_080_000, 4008, 4016            # (rows of 4008 codes are copied first, rows of 4016 are not)
F64 = torch.float64


def far_rows(rows, cols):
    r = [0, 1, rows - 2, rows - 1]
    for at in (1 << 30, 1 << 31, 1 << 32):
        if at // cols + 1 < rows:
            r += [at // cols - 1, at // cols, at // cols + 1]
    return torch.tensor(sorted(set(r)), device="cuda")


def few(seed, rows, cols, most=2):
    """zero but in the far rows; the rows differ"""
    t = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    at = far_rows(rows, cols)
    t[at] = whole(seed, len(at), cols, BF16, most)
    return t, at


def same(got, want, lo=0):
    assert torch.equal(got[lo:lo + want.shape[0]], want.to(BF16)), lo


def values(q, scale):
    """what codes (a block of rows) and their scales (blocks of columns, rows) stand for"""
    s = torch.exp2(scale.view(torch.uint8).to(F32) - 127).t().repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.to(F32) * s


@pytest.mark.parametrize("rows", [1, 128])
def test_quantiser(tfla, rows):  # noqa: F811
    print("far quantiser", rows, flush=True)
    x = whole(1, M, WIDE, BF16)
    o = tfla.q8_quant(x, rows=rows, want_t=True)
    for lo in range(0, M, 64_000):
        hi = min(M, lo + 64_000)
        per = rows if rows > 1 else 1
        s = o["scale"][:, lo // per:-(-hi // per)].view(torch.uint8).repeat_interleave(per, 1)[:, :hi - lo]
        assert torch.equal(values(o["q"][lo:hi], s), x[lo:hi].float()), lo
        st = o["scale_t"][lo // 128:-(-hi // 128)].view(torch.uint8).repeat_interleave(per, 1)[:, :WIDE]
        st = torch.exp2(st.to(F32) - 127).repeat_interleave(128, 0)[:hi - lo]
        assert torch.equal(o["qt"][:, lo:hi].t().to(F32) * st, x[lo:hi].float()), lo


def test_norm(tfla):  # noqa: F811
    """every row is its own: against calls of some rows at a time"""
    print("far norm", flush=True)
    x, r = whole(2, M, WIDE, BF16), whole(3, M, WIDE, BF16)
    o = tfla.norm_q8_fwd(x, residual=r, keep_y=True)
    for lo, hi in blocks(M):
        p = tfla.norm_q8_fwd(x[lo:hi], residual=r[lo:hi], keep_y=True)
        for k in ("q", "sum", "y", "rstd"):
            assert torch.equal(o[k][lo:hi].view(torch.uint8), p[k].view(torch.uint8)), (k, lo)
        assert torch.equal(o["scale"][:, lo:hi].view(torch.uint8), p["scale"].view(torch.uint8)), lo


@pytest.mark.parametrize("K", [WIDE, EVEN])
def test_forward_input(tfla, K):  # noqa: F811
    print("far forward input", K, flush=True)
    x, w = whole(4, M, K, BF16, 1), torch.zeros((40, K), dtype=BF16, device="cuda")
    w[:, ::37] = whole(5, 40, (K + 36) // 37, BF16, 1)
    xq, wq = tfla.q8_quant(x), tfla.q8_quant(w, rows=128)
    y = tfla.linear_q8_fwd(xq["q"], xq["scale"], wq["q"], wq["scale"])["y"]
    for lo, hi in blocks(M):
        same(y, x[lo:hi].double() @ w.double().t(), lo)


def test_forward_results(tfla):  # noqa: F811
    """y, z, hq, h_scale, h, a and u written, the residual read"""
    print("far forward results", flush=True)
    x, w = whole(6, M, 32, BF16), whole(7, WIDE, 32, BF16, 1)
    res = whole(8, M, WIDE, BF16)
    xq, wq = tfla.q8_quant(x), tfla.q8_quant(w, rows=128)
    f = tfla.linear_q8_fwd(xq["q"], xq["scale"], wq["q"], wq["scale"], residual=res, act=tfla.ACT_RELU, keep_pre=True)
    for lo, hi in blocks(M):
        z = x[lo:hi].double() @ w.double().t()
        same(f["z"], z, lo)
        same(f["y"], z.clamp_min(0) + res[lo:hi].double(), lo)
    del f, res
    # (sums of three products of ones: h is at most 9 and a code)
    w2 = whole(9, WIDE, 32, BF16, 1)
    w2[:, 3:] = 0
    w[:, 3:] = 0
    x.clamp_(-1, 1)
    xq, wq, w2q = tfla.q8_quant(x), tfla.q8_quant(w, rows=128), tfla.q8_quant(w2, rows=128)
    f = tfla.gated_q8_fwd(xq["q"], xq["scale"], wq["q"], wq["scale"], w2q["q"], w2q["scale"], act=tfla.ACT_RELU, keep_pre=True)
    for lo, hi in blocks(M):
        a, u = (x[lo:hi].double() @ t.double().t() for t in (w, w2))
        same(f["a"], a, lo)
        same(f["u"], u, lo)
        h = a.clamp_min(0) * u
        same(f["h"], h, lo)
        assert torch.equal(values(f["hq"][lo:hi], f["h_scale"][:, lo:hi]), h.float()), lo


@pytest.mark.parametrize("N", [WIDE, EVEN])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_backward_gradients_of_results(tfla, act, N):  # noqa: F811
    """dy and z read, their gradient's codes written and read as either operand, the bias sums"""
    print("far backward results", act, N, flush=True)
    K = 64
    dy, at = few(10, M, N)
    x, w = whole(11, M, K, BF16), torch.zeros((N, K), dtype=BF16, device="cuda")
    w[::37] = whole(12, (N + 36) // 37, K, BF16, 1)
    wq = tfla.q8_quant(w, rows=128, want_t=True)
    dz, z = dy[at].double(), None
    if act == "relu":
        z = whole(13, M, N, BF16)
        dz = dz * (z[at] > 0)
    g = tfla.linear_q8_bwd(x, wq["qt"], wq["scale_t"], dy, z, act=tfla.ACT_RELU if z is not None else tfla.ACT_NONE, want_db=True)
    same(g["dw"], dz.t() @ x[at].double())
    assert torch.equal(g["db"].double(), dz.sum(0))
    same(g["dx"][at], dz @ w.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


def test_backward_of_the_pair(tfla):  # noqa: F811
    print("far backward pair", flush=True)
    K, N = 64, WIDE
    dh, at = few(14, M, N)
    x = whole(15, M, K, BF16, 1)
    wg, wu = (torch.zeros((N, K), dtype=BF16, device="cuda") for _ in range(2))
    wg[::97], wu[1::97] = whole(16, len(range(0, N, 97)), K, BF16, 1), whole(17, len(range(1, N, 97)), K, BF16, 1)
    a, u = whole(18, M, N, BF16), whole(19, M, N, BF16)
    gq, uq = tfla.q8_quant(wg, rows=128, want_t=True), tfla.q8_quant(wu, rows=128, want_t=True)
    g = tfla.gated_q8_bwd(x, gq["qt"], gq["scale_t"], uq["qt"], uq["scale_t"], a, u, dh, act=tfla.ACT_RELU, want_db=True)
    d, av, uv = dh[at].double(), a[at].double(), u[at].double()
    da, du = d * uv * (av > 0), d * av.clamp_min(0)
    same(g["dw_gate"], da.t() @ x[at].double())
    same(g["dw_up"], du.t() @ x[at].double())
    assert torch.equal(g["db_gate"].double(), da.sum(0)) and torch.equal(g["db_up"].double(), du.sum(0))
    same(g["dx"][at], da @ wg.double() + du @ wu.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


def test_backward_gradients_of_inputs(tfla):  # noqa: F811
    """dx written; x read, its transpose's codes written and read"""
    print("far backward inputs", flush=True)
    N, K = 40, WIDE
    at = far_rows(M, K)
    x, w, dy = whole(20, M, K, BF16), whole(21, N, K, BF16, 1), torch.zeros((M, N), dtype=BF16, device="cuda")
    dy[at] = whole(22, len(at), N, BF16)
    wq = tfla.q8_quant(w, rows=128, want_t=True)
    g = tfla.linear_q8_bwd(x, wq["qt"], wq["scale_t"], dy)
    same(g["dw"], dy[at].double().t() @ x[at].double())
    same(g["dx"][at], dy[at].double() @ w.double())
    g["dx"][at] = 0
    assert not g["dx"].any()


@pytest.mark.parametrize("K", [4104, 4112])
@pytest.mark.parametrize("tokens", [2, 40])
def test_weights(tfla, tokens, K):  # noqa: F811
    """weights, their transpose and their gradients, by the kernel for few rows and by tiles"""
    print("far weights", tokens, K, flush=True)
    N = 1_048_560 if K % 16 == 0 else 1 << 20
    x = torch.zeros((tokens, K), dtype=BF16, device="cuda")
    x[:, ::37] = whole(23, tokens, (K + 36) // 37, BF16, 1)
    w, at = few(24, N, K)
    wq, xq = tfla.q8_quant(w, rows=128, want_t=True), tfla.q8_quant(x)
    y = tfla.linear_q8_fwd(xq["q"], xq["scale"], wq["q"], wq["scale"])["y"]
    want = x.double() @ w[at].double().t()
    same(y[:, at], want)
    y[:, at] = 0
    assert not y.any()
    o = tfla.gated_q8_fwd(xq["q"], xq["scale"], wq["q"], wq["scale"], wq["q"], wq["scale"], act=tfla.ACT_RELU, keep_pre=True)
    same(o["h"][:, at], want.clamp_min(0) * want)
    o["h"][:, at] = 0
    assert not o["h"].any()
    del o
    dy = torch.zeros((tokens, N), dtype=BF16, device="cuda")
    dy[:, at] = whole(25, tokens, len(at), BF16, 1)
    g = tfla.linear_q8_bwd(x, wq["qt"], wq["scale_t"], dy)
    same(g["dx"], dy[:, at].double() @ w[at].double())
    same(g["dw"][at], dy[:, at].double().t() @ x.double())
    g["dw"][at] = 0
    assert not g["dw"].any()
